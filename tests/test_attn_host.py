"""Host-side checks of the operators around an attention layer that need no
GPU: arguments that the C ABI refuses before anything is enqueued, the shapes
and types that the binding refuses, workspace sizes, rotary frequencies."""
import ctypes
import math

import pytest
import torch

import paper_1907_00641_amd as P
from paper_1907_00641_amd import binding as B

FAKE = [ctypes.c_void_p(0x100000000 * (i + 1)) for i in range(16)]  # far apart, never read
BAD = B.PAM_ERR_INVALID_ARGUMENT


@pytest.fixture(scope="module")
def L():
    import os

    if not os.path.exists(B.LIB_PATH):
        from paper_1907_00641_amd.build import build_library

        build_library()
    return B.lib()


def attn_desc(**over):
    f = dict(dtype=2, batch=2, heads=4, kv_heads=2, dim=8, dim_v=16, len_q=5, len_k=6, flags=0, scale=0.5)
    f.update({k: v for k, v in over.items() if not k.endswith("stride")})
    H, hk, d, dv, lq, lk = (f[x] for x in ("heads", "kv_heads", "dim", "dim_v", "len_q", "len_k"))
    strides = dict(q_stride=(lq * H * 2 * d, H * 2 * d, 2 * d, d), k_stride=(lk * hk * 2 * d, hk * 2 * d, 2 * d, d),
                   v_stride=(lk * hk * dv, hk * dv, dv))
    strides.update({k: v for k, v in over.items() if k.endswith("stride")})
    return B.DiffAttnDesc(**f, **strides)


@pytest.mark.parametrize("over", [dict(dtype=3), dict(dtype=-1), dict(batch=-1), dict(heads=0), dict(kv_heads=0),
                                  dict(kv_heads=3), dict(dim=0), dict(dim=129), dict(dim_v=0), dict(dim_v=257),
                                  dict(len_q=-1), dict(len_k=-1), dict(flags=2), dict(scale=0.0), dict(scale=-1.0),
                                  dict(scale=math.inf), dict(scale=math.nan), dict(len_q=2 ** 31 - 1),
                                  dict(batch=2 ** 16, heads=2 ** 14, kv_heads=2 ** 14, len_q=2 ** 8),
                                  dict(q_stride=(2 ** 62, 1, 1, 1)), dict(v_stride=(1, -2 ** 62, 1))],
                         ids=lambda o: "-".join(f"{k}={v}" for k, v in o.items())[:40])
def test_attention_refuses(L, over):
    d = attn_desc(**over)
    assert L.pam_diff_attn_fwd(ctypes.byref(d), *FAKE[:4], None, None, None, FAKE[4], None, None, FAKE[5], None) == BAD
    assert B.last_error()
    assert L.pam_diff_attn_bwd(ctypes.byref(d), *FAKE[:4], None, None, None, *FAKE[4:7], (ctypes.c_int64 * 3)(1, 1, 1),
                               *FAKE[7:12], None) == BAD
    if not any(k.endswith("stride") for k in over):
        assert L.pam_diff_attn_fwd_workspace(ctypes.byref(d)) == ctypes.c_size_t(-1).value
        assert L.pam_diff_attn_bwd_workspace(ctypes.byref(d)) == ctypes.c_size_t(-1).value


def test_attention_refuses_pointers(L):
    d = ctypes.byref(attn_desc())
    q, k, v, lam, out, so, lse = FAKE[:7]
    ok = [q, k, v, lam, None, None, None, out, None, None, None, None]
    for i in (0, 1, 2, 3, 7):
        args = list(ok)
        args[i] = None
        assert L.pam_diff_attn_fwd(d, *args) == BAD, i
    assert L.pam_diff_attn_fwd(None, *ok) == BAD
    assert L.pam_diff_attn_fwd(d, q, k, v, lam, None, None, None, out, so, None, None, None) == BAD  # lse missing
    assert "together" in B.last_error()
    assert L.pam_diff_attn_fwd(d, q, k, v, lam, None, None, None, q, None, None, None, None) == BAD  # in place
    assert L.pam_diff_attn_fwd(d, q, k, v, lam, None, None, None, out, out, lse, None, None) == BAD
    strides = (ctypes.c_int64 * 3)(1, 1, 1)
    good = [q, k, v, lam, None, None, None, so, lse, FAKE[7], strides, *FAKE[8:13], None]
    for i in (0, 1, 2, 3, 7, 8, 9, 10, 11, 12, 13, 14, 15):
        args = list(good)
        args[i] = None
        assert L.pam_diff_attn_bwd(d, *args) == BAD, i
    good[15] = ctypes.c_void_p(FAKE[12].value + 4)  # workspace not aligned
    assert L.pam_diff_attn_bwd(d, *good) == BAD
    # no queries: nothing is done and nothing is needed
    assert L.pam_diff_attn_fwd(ctypes.byref(attn_desc(len_q=0)), *([None] * 12)) == B.PAM_OK


def test_rotary_refuses(L):
    ok = dict(dtype=1, batch=1, length=3, heads=2, kv_heads=1, dim=8, pairs=4, flags=0, start=0, entries=9,
              q_stride=(48, 16, 8), k_stride=(24, 8, 8))

    def call(args=FAKE[:6], **over):
        d = B.RotaryDesc(**{**ok, **over})
        q, k, t, p, qo, ko = args
        return L.pam_rotary(ctypes.byref(d), q, k, t, p, qo, ko, None)

    for over in (dict(dtype=5), dict(batch=-1), dict(length=-1), dict(heads=0), dict(kv_heads=-1), dict(dim=0),
                 dict(dim=1025), dict(pairs=0), dict(pairs=5), dict(flags=4), dict(entries=0), dict(entries=-1),
                 dict(start=-2 ** 63), dict(batch=2 ** 30, length=2 ** 10), dict(q_stride=(1, 2 ** 62, 1))):
        assert call(**over) == BAD, over
    for i in (0, 1, 2, 4, 5):
        args = list(FAKE[:6])
        args[i] = None
        assert call(args) == BAD, i
    q, k, t, p, qo, ko = FAKE[:6]
    assert call((q, k, t, p, q, ko), q_stride=(60, 20, 8)) == BAD  # in place, not contiguous
    assert call((q, k, t, p, ctypes.c_void_p(q.value + 16), ko)) == BAD
    assert call((q, k, t, p, k, ko)) == BAD
    assert call((q, k, ctypes.c_void_p(t.value + 4), p, qo, ko)) == BAD
    assert L.pam_rotary(None, *FAKE[:6], None) == BAD
    assert call(batch=0) == B.PAM_OK
    f = FAKE
    for pairs, axes, entries, coord, mag in ((0, 1, 4, None, 1.0), (257, 1, 4, None, 1.0), (4, 0, 4, f[1], 1.0),
                                             (4, 17, 4, f[1], 1.0), (4, 2, 4, None, 1.0), (4, 1, -1, None, 1.0),
                                             (4, 1, 2 ** 30, None, 1.0), (4, 1, 4, None, math.inf)):
        assert L.pam_rotary_table(f[0], coord, None, entries, pairs, axes, mag, f[2], None) == BAD
    assert L.pam_rotary_table(None, None, None, 4, 4, 1, 1.0, f[2], None) == BAD
    assert L.pam_rotary_table(f[0], None, None, 4, 4, 1, 1.0, None, None) == BAD


def test_rotary_frequencies():
    f, mag = P.pam_rotary_frequencies(8, 10000.0)
    want = torch.tensor([10000.0 ** (-2 * i / 8) for i in range(4)], dtype=torch.float64)
    assert mag == 1.0 and torch.allclose(f, want, rtol=1e-14, atol=0)
    lin, mag = P.pam_rotary_frequencies(8, 10000.0, "linear", 4.0)
    assert mag == 1.0 and torch.allclose(lin, want / 4, rtol=1e-14, atol=0)
    # the fastest pair as it was, the slowest stretched by the factor
    ntk, mag = P.pam_rotary_frequencies(8, 10000.0, "ntk", 4.0)
    assert mag == 1.0 and ntk[0] == want[0] and abs(ntk[3] * 4 / want[3] - 1) < 1e-13
    # by parts: over 2048 positions the pairs turn 2048 f / 2 pi times
    y, mag = P.pam_rotary_frequencies(64, 10000.0, "yarn", 8.0, 2048.0)
    plain, _ = P.pam_rotary_frequencies(64, 10000.0)
    turns = 2048.0 * plain / (2 * math.pi)
    assert mag == pytest.approx(0.1 * math.log(8.0) + 1.0, rel=1e-15)
    assert torch.equal(y[turns > 32], plain[turns > 32])
    assert torch.allclose(y[turns < 1], plain[turns < 1] / 8, rtol=1e-14, atol=0)
    part = (turns >= 1) & (turns <= 32)
    g = (turns[part] - 1) / 31
    assert part.any() and torch.allclose(y[part], ((1 - g) / 8 + g) * plain[part], rtol=1e-13, atol=0)
    for bad in ((7,), (0,), (514,), (8, 1.0), (8, math.nan), (8, 1e4, "linear", 0.5), (2, 1e4, "ntk", 2.0),
                (8, 1e4, "yarn", 2.0, 0.0), (8, 1e4, "yarn", 2.0, 10.0, 3.0, 2.0)):
        with pytest.raises(P.PamError):
            P.pam_rotary_frequencies(*bad)
    with pytest.raises(ValueError):
        P.pam_rotary_frequencies(8, 1e4, "other")


def test_dropout_refuses(L):
    x, y = FAKE[:2]
    for n, t, p in ((-1, 0, 0.1), (2 ** 40, 0, 0.1), (4, 3, 0.1), (4, 0, -0.1), (4, 0, 1.1), (4, 0, math.nan)):
        assert L.pam_dropout(x, n, t, p, 1, 1, y, None) == BAD
    assert L.pam_dropout(None, 4, 0, 0.1, 1, 1, y, None) == BAD
    assert L.pam_dropout(x, 4, 0, 0.1, 1, 1, None, None) == BAD
    assert L.pam_dropout(x, 4, 0, 0.1, 1, 1, ctypes.c_void_p(x.value + 4), None) == BAD
    assert L.pam_dropout(None, 0, 0, 0.1, 1, 1, None, None) == B.PAM_OK


def test_norm_refuses(L):
    ok = dict(dtype=2, norm=0, rows=6, channels=16, eps=1e-6, gate_rows=2, x_stride=16, z_stride=16, p=0.1, seed=1,
              offset=1)
    x, z, wq, bq, g, sc, wp, bp, r, h = FAKE[:10]

    def fwd(args=(x, z, wq, bq, g, sc, wp, bp, r, h), **over):
        return L.pam_norm_gate_fwd(ctypes.byref(B.NormDesc(**{**ok, **over})), *args, None)

    for over in (dict(dtype=4), dict(norm=2), dict(rows=-1), dict(channels=0), dict(channels=8193), dict(eps=-1.0),
                 dict(eps=math.nan), dict(p=1.5), dict(gate_rows=4), dict(gate_rows=0), dict(rows=2 ** 40),
                 dict(x_stride=2 ** 61)):
        assert fwd(**over) == BAD, over
    assert fwd((None, z, wq, bq, g, sc, wp, bp, r, h)) == BAD
    assert fwd((x, None, wq, bq, g, sc, wp, bp, r, h)) == BAD        # gate without z
    assert fwd((x, None, None, None, None, None, wp, bp, r, h)) == BAD  # r without z
    assert fwd((x, z, wq, bq, g, sc, wp, bp, None, h)) == BAD        # z without r
    assert fwd((x, z, wq, bq, g, sc, wp, bp, r, None)) == BAD        # w_pre without h
    assert fwd((x, None, None, None, None, None, None, None, None, None)) == BAD
    assert fwd((x, z, wq, bq, g, sc, wp, bp, r, r)) == BAD
    assert fwd((x, z, wq, bq, g, sc, wp, bp, r, x)) == BAD
    assert fwd((x, z, wq, bq, g, sc, wp, bp, x, h), x_stride=20) == BAD
    assert fwd(rows=0) == B.PAM_OK
    gr, gh, gx, gz, gwq, ws = FAKE[10:16]

    def bwd(args, **over):
        return L.pam_norm_gate_bwd(ctypes.byref(B.NormDesc(**{**ok, **over})), *args, None)

    good = [x, z, wq, bq, g, sc, wp, gr, gh, gx, gz, gwq, None, None, None, None, None, ws]
    for i in (0, 1, 17):
        args = list(good)
        args[i] = None
        assert bwd(args) == BAD, i
    for i, bad in ((8, None), (9, gh), (9, x), (10, gx), (17, ctypes.c_void_p(ws.value + 8))):
        args = list(good)
        args[i] = bad
        assert bwd(args) == BAD, i
    assert bwd([x, z, None, None, None, None, wp, gr, gh, gx, gz, None, None, gwq, None, None, None, ws]) == BAD
    assert bwd(good, gate_rows=4) == BAD
    assert L.pam_norm_gate_bwd_workspace(ctypes.byref(B.NormDesc(**{**ok, "gate_rows": 4}))) == ctypes.c_size_t(-1).value
    assert L.pam_norm_gate_bwd_workspace(ctypes.byref(B.NormDesc(**ok))) >= 5 * 16 * 4


def test_binding_refuses_cpu_tensors_and_shapes():
    q = torch.zeros(1, 2, 2, 2, 8)
    with pytest.raises(ValueError, match="device"):
        P.pam_diff_attn_fwd(q, q, q[:, :, :, 0], torch.zeros(2))
    with pytest.raises(ValueError, match="B x Lq"):
        P.pam_diff_attn_fwd(q[0], q, q[:, :, :, 0], torch.zeros(2))
    with pytest.raises(ValueError, match="agree"):
        P.pam_diff_attn_fwd(q, q[:, :1], q[:, :, :, 0], torch.zeros(2))
    with pytest.raises(ValueError, match="float32"):
        P.pam_diff_attn_fwd(q.double(), q, q[:, :, :, 0], torch.zeros(2))
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device"):
        P.pam_dropout(x, 0.1, 1)
    with pytest.raises(ValueError, match="device"):
        P.pam_norm_gate_fwd(x)
    with pytest.raises(ValueError, match="rows x channels"):
        P.pam_norm_gate_fwd(x, z=x[:2])
    with pytest.raises(ValueError, match="norm must"):
        P.pam_norm_gate_fwd(x, norm="batch")
    with pytest.raises(ValueError, match="dividing"):
        P.pam_norm_gate_fwd(x, z=x, gate=torch.zeros(3, 8))
    with pytest.raises(ValueError, match="B x L"):
        P.pam_rotary(q, None, torch.zeros(4, 4, 2))
    with pytest.raises(ValueError, match="pairs x 2"):
        P.pam_rotary(q[0], None, torch.zeros(4, 8))
    with pytest.raises(ValueError, match="entries or coord"):
        P.pam_rotary_table(torch.zeros(4, dtype=torch.float64))
