"""Host-side checks of attention over packed sequences and from a paged cache that need no GPU: arguments that the C
ABI refuses before anything is enqueued, what the binding refuses, workspace sizes."""
import ctypes
import math

import pytest
import torch

import paper_1907_00641_amd as P
from paper_1907_00641_amd import binding as B
from test_attn_host import BAD, FAKE, L  # noqa: F401

FAR = (1 << 32) + 5


def at(p, off):
    return ctypes.c_void_p(p.value + off)


def made(kind, ok, over):
    return kind(**{**ok, **over})


ATTN = dict(dtype=2, sequences=2, heads=4, kv_heads=2, dim=8, dim_v=16, flags=0, scale=0.5, tokens=5, keys=6,
            q_stride=(32, 8), k_stride=(16, 8), v_stride=(32, 16))


@pytest.mark.parametrize("over", [dict(dtype=3), dict(sequences=0), dict(sequences=-1), dict(heads=0), dict(kv_heads=3),
                                  dict(kv_heads=0), dict(dim=0), dict(dim=129), dict(dim_v=0), dict(dim_v=129),
                                  dict(flags=2), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf),
                                  dict(tokens=-1), dict(keys=-1), dict(tokens=2 ** 30), dict(keys=2 ** 30),
                                  dict(tokens=2 ** 29, heads=4), dict(sequences=2 ** 23, heads=2 ** 6),
                                  dict(q_stride=(2 ** 62, 1)), dict(v_stride=(1, -2 ** 62))],
                         ids=lambda o: "-".join(f"{k}={v}" for k, v in o.items())[:40])
def test_attention_refuses(L, over):
    d = ctypes.byref(made(B.AttnDesc, ATTN, over))
    f = FAKE
    assert L.pam_attn_fwd(d, *f[:6], None, None, f[6], None) == BAD and B.last_error()
    assert L.pam_attn_bwd(d, *f[:8], (ctypes.c_int64 * 2)(1, 1), *f[8:12], None) == BAD
    if not any(k.endswith("stride") for k in over):
        assert L.pam_attn_fwd_workspace(d) == ctypes.c_size_t(-1).value
        assert L.pam_attn_bwd_workspace(d) == ctypes.c_size_t(-1).value


def test_attention_refuses_pointers(L):
    d = ctypes.byref(made(B.AttnDesc, ATTN, {}))
    q, k, v, qs, ks, out, so, lse, ws = FAKE[:9]
    good = [q, k, v, qs, ks, out, so, lse, ws, None]
    for i in (0, 1, 2, 3, 4, 5, 6, 7):
        args = list(good)
        args[i] = None
        assert L.pam_attn_fwd(d, *args) == BAD, i
    for i, bad in ((5, q), (5, at(ks, 8)), (6, v), (7, at(qs, 0)), (6, out)):
        args = list(good)
        args[i] = bad
        assert L.pam_attn_fwd(d, *args) == BAD and "overlap" in B.last_error(), (i, bad)
    assert L.pam_attn_fwd(None, *good) == BAD
    f = FAKE
    good = [q, k, v, qs, ks, so, lse, f[8], (ctypes.c_int64 * 2)(64, 16), f[9], f[10], f[11], f[12], None]
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12):
        args = list(good)
        args[i] = None
        assert L.pam_attn_bwd(d, *args) == BAD, i
    for i, bad in ((9, f[8]), (10, f[9]), (11, so), (12, at(f[12], 8)), (12, q)):
        args = list(good)
        args[i] = bad
        assert L.pam_attn_bwd(d, *args) == BAD, (i, bad)
    # no queries: nothing is done and nothing is needed
    assert L.pam_attn_fwd(ctypes.byref(made(B.AttnDesc, ATTN, dict(tokens=0))), *([None] * 10)) == B.PAM_OK


def test_attention_workspaces(L):
    """Parts are cut where the units do not fill the card, and only there."""
    few = made(B.AttnDesc, ATTN, dict(sequences=1, heads=2, kv_heads=1, dim=64, dim_v=64, tokens=2000, keys=2000))
    many = made(B.AttnDesc, ATTN, dict(sequences=1, heads=64, kv_heads=8, dim=64, dim_v=64, tokens=20000, keys=20000))
    assert 0 < L.pam_attn_fwd_workspace(ctypes.byref(few)) < 2 ** 28
    assert L.pam_attn_fwd_workspace(ctypes.byref(many)) == 0
    assert L.pam_attn_bwd_workspace(ctypes.byref(many)) >= 2 * 64 * 20000 * 4


NORM = dict(dtype=1, norm=0, batch=1, length=3, heads=2, kv_heads=1, dim=8, pairs=4, flags=0, w_per_head=0, eps=1e-6,
            start=0, entries=9, q_stride=(48, 16, 8), k_stride=(24, 8, 8))


def test_head_norm_refuses(L):
    q, k, wq, wk, t, p, qo, ko = FAKE[:8]

    def fwd(args=(q, k, wq, wk, t, p, qo, ko), **over):
        return L.pam_head_norm_rotary_fwd(ctypes.byref(made(B.HeadNormDesc, NORM, over)), *args, None)

    for over in (dict(dtype=5), dict(norm=2), dict(batch=-1), dict(length=-1), dict(heads=0), dict(kv_heads=-1),
                 dict(dim=0), dict(dim=513), dict(pairs=0), dict(pairs=5), dict(flags=2), dict(eps=-1.0),
                 dict(eps=math.nan), dict(entries=0), dict(entries=-1), dict(start=2 ** 62),
                 dict(batch=2 ** 20, length=2 ** 10), dict(q_stride=(1, 2 ** 62, 1))):
        assert fwd(**over) == BAD, over
    for i in (0, 1, 4, 6, 7):
        args = [q, k, wq, wk, t, p, qo, ko]
        args[i] = None
        assert fwd(args) == BAD, i
    assert fwd((q, k, wq, wk, t, p, q, ko), q_stride=(60, 20, 8)) == BAD  # in place, not contiguous
    for bad in (at(q, 16), k, at(wq, 28), at(wk, 0), at(t, 9 * 4 * 8 - 8), at(p, 8)):
        assert fwd((q, k, wq, wk, t, p, bad, ko)) == BAD, bad
        assert fwd((q, k, wq, wk, t, p, qo, at(bad, 0) if bad is not k else q)) == BAD, bad
    assert fwd((q, k, wq, wk, at(t, 4), p, qo, ko)) == BAD
    assert fwd(batch=0) == B.PAM_OK
    assert L.pam_head_norm_rotary_fwd(None, q, k, wq, wk, t, p, qo, ko, None) == BAD
    gq, gk, dq, dk, dwq, dwk, ws = FAKE[8:15]

    def bwd(args, **over):
        return L.pam_head_norm_rotary_bwd(ctypes.byref(made(B.HeadNormDesc, NORM, over)), *args, None)

    good = [q, k, wq, wk, t, p, gq, gk, dq, dk, dwq, dwk, ws]
    for i in (0, 1, 4, 6, 7, 8, 9, 12):
        args = list(good)
        args[i] = None
        assert bwd(args) == BAD, i
    for i, bad in ((8, q), (8, gk), (9, gq), (10, wq), (11, dwq), (8, at(gq, 8)), (12, at(ws, 8)), (12, t), (10, dq)):
        args = list(good)
        args[i] = bad
        assert bwd(args) == BAD, (i, bad)
    d = ctypes.byref(made(B.HeadNormDesc, NORM, dict(dim=600)))
    assert L.pam_head_norm_rotary_bwd_workspace(d) == ctypes.c_size_t(-1).value


CACHE = dict(dtype=2, store=3, pages=6, page_size=4, kv_heads=2, dim=8, dim_v=16, maps=1, sequences=2, table_width=3)
CACHE_BAD = (dict(dtype=3), dict(store=5), dict(store=1), dict(store=-1), dict(pages=-1), dict(page_size=0),
             dict(kv_heads=0), dict(dim=0), dict(dim=257), dict(dim=129, maps=2), dict(dim_v=0), dict(dim_v=257),
             dict(maps=0), dict(maps=3), dict(sequences=-1), dict(table_width=-1), dict(pages=2 ** 30),
             dict(table_width=2 ** 28))


def test_cache_refuses(L):
    k, v, new, t, n, kp, vp, ks, vs = FAKE[:9]
    rows = dict(rows=0, length=3, k_stride=(48, 16, 8, 0), v_stride=(96, 32, 16))

    def write(args=(k, v, None, new, t, n, kp, vp, ks, vs), r=rows, **over):
        return L.pam_cache_write(ctypes.byref(made(B.CacheDesc, CACHE, over)), ctypes.byref(B.CacheRows(**r)), *args, None)

    def read(args=(t, n, kp, vp, ks, vs, k, v), length=5, **over):
        return L.pam_cache_read(ctypes.byref(made(B.CacheDesc, CACHE, over)), length, *args, None)

    for over in CACHE_BAD:
        assert write(**over) == BAD, over
        assert read(**over) == BAD, over
    for i in (0, 1, 4, 5, 6, 7, 8, 9):
        args = [k, v, None, new, t, n, kp, vp, ks, vs]
        args[i] = None
        assert write(args) == BAD, i
    assert write((k, v, FAKE[9], new, t, n, kp, vp, ks, vs)) == BAD  # starts and new_len
    assert write((k, v, None, new, t, n, at(kp, 8), vp, ks, vs)) == BAD
    assert write(store=2) == BAD and "8 bits" in B.last_error()  # scales
    for over in (dict(length=-1), dict(length=2 ** 30 + 1), dict(k_stride=(2 ** 62, 1, 1, 1))):
        assert write(r={**rows, **over}) == BAD, over
    assert write((k, v, FAKE[9], None, t, n, kp, vp, ks, vs), r={**rows, "rows": -1}) == BAD
    for i, bad in ((6, k), (7, v), (8, at(new, 4)), (9, at(t, 20)), (6, at(n, 0)), (7, kp), (9, ks)):
        args = [k, v, None, new, t, n, kp, vp, ks, vs]
        args[i] = bad
        if i in (6, 7):
            args[i] = ctypes.c_void_p(bad.value // 16 * 16)
        assert write(args) == BAD and "overlap" in B.last_error(), (i, bad)
    assert write(sequences=0) == B.PAM_OK and write(r={**rows, "length": 0}) == B.PAM_OK
    for i in (0, 1, 2, 3, 4, 5):
        args = [t, n, kp, vp, ks, vs, k, v]
        args[i] = None
        assert read(args) == BAD, i
    assert read(length=-1) == BAD
    for i, bad in ((6, kp), (7, at(ks, 4)), (7, at(t, 0)), (7, k), (6, at(k, 1))):
        args = [t, n, kp, vp, ks, vs, k, v]
        args[i] = bad
        assert read(args) == BAD, (i, bad)
    assert read(length=0) == B.PAM_OK and read((t, n, kp, vp, ks, vs, None, None)) == B.PAM_OK


PAGED = dict(heads=4, len_q=3, key_bound=0, scale=0.5, q_stride=(96, 32, 8, 0))


def test_paged_attention_refuses(L):
    q, lam, ql, t, n, kp, vp, ks, vs, out, ws = FAKE[:11]
    good = [q, None, ql, t, n, kp, vp, ks, vs, out, ws]

    def call(args=good, cache={}, **over):
        return L.pam_paged_attn(ctypes.byref(made(B.CacheDesc, CACHE, cache)),
                                ctypes.byref(made(B.PagedAttnDesc, PAGED, over)), *args, None)

    none = ctypes.c_size_t(-1).value
    for over in CACHE_BAD:
        assert call(cache=over) == BAD, over
        assert L.pam_paged_attn_workspace(ctypes.byref(made(B.CacheDesc, CACHE, over)),
                                          ctypes.byref(made(B.PagedAttnDesc, PAGED, {}))) == none
    for over in (dict(heads=0), dict(heads=3), dict(len_q=-1), dict(len_q=2 ** 20), dict(key_bound=-1), dict(scale=0.0),
                 dict(scale=math.nan), dict(q_stride=(2 ** 62, 1, 1, 1))):
        assert call(**over) == BAD, over
    assert call(cache=dict(sequences=2 ** 15), heads=2 ** 10, len_q=2 ** 10) == BAD
    # rows of both maps and units are numbers of 32 bits
    for over, cache in ((dict(heads=2 ** 11, len_q=2 ** 19), dict(maps=2)), (dict(heads=2 ** 12, len_q=2 ** 19 - 1), dict(maps=1)),
                        (dict(heads=2 ** 16, len_q=1), dict(sequences=2 ** 15 - 1))):
        assert call(cache=cache, **over) == BAD and "2^30" in B.last_error()
        assert L.pam_paged_attn_workspace(ctypes.byref(made(B.CacheDesc, CACHE, cache)),
                                          ctypes.byref(made(B.PagedAttnDesc, PAGED, over))) == none
    for i in (0, 3, 4, 5, 6, 7, 8, 9):
        args = list(good)
        args[i] = None
        assert call(args) == BAD, i
    assert call([q, lam, *good[2:]]) == BAD and "two maps" in B.last_error()
    assert call(good, cache=dict(maps=2)) == BAD and "two maps" in B.last_error()
    for bad in (q, at(ql, 4), at(t, 0), at(n, 4), at(kp, 100), vp, at(ks, 8), vs):
        args = list(good)
        args[9] = bad
        assert call(args) == BAD and "overlap" in B.last_error(), bad
    assert call(len_q=0) == B.PAM_OK
    long = dict(pages=4096, page_size=16, table_width=2048)
    c, d = ctypes.byref(made(B.CacheDesc, CACHE, long)), ctypes.byref(made(B.PagedAttnDesc, PAGED, {}))
    assert 0 < L.pam_paged_attn_workspace(c, d) < 2 ** 26
    args = list(good)
    for bad in (None, at(ws, 4), q):
        args[10] = bad
        assert call(args, cache=long) == BAD, bad
    short = ctypes.byref(made(B.PagedAttnDesc, PAGED, dict(key_bound=30)))
    assert L.pam_paged_attn_workspace(c, short) == 0


def one(*shape):
    return torch.zeros(1).as_strided(shape, (0,) * len(shape))


def test_binding_refuses():
    q = torch.zeros(5, 2, 8)
    s = torch.zeros(3, dtype=torch.int32)
    for args, how, text in (((q, q, q), {}, "device"), ((q[0], q, q), {}, "T x H"), ((q, q[:2], q), {}, "agree"),
                            ((q, q, q), dict(q_start=s), "together"), ((q.double(), q, q), {}, "float32"),
                            ((q, q, q), dict(q_start=s[:1], k_start=s[:1]), "one more"),
                            ((one(FAR, 2, 8), q, q), {}, r"2\^31"), ((q, one(FAR, 2, 8), one(FAR, 2, 8)), {}, r"2\^31")):
        with pytest.raises(ValueError, match=text):
            P.pam_attn_fwd(*args, **how)
        with pytest.raises(ValueError, match=text):
            P.pam_attn_bwd(*args, (None, None), q, **how)
    x, table = torch.zeros(1, 2, 2, 8), torch.zeros(4, 4, 2)
    w = torch.ones(8)
    for args, how, text in (((x, None, table), {}, "device"), ((x[0], None, table), {}, "B x L"),
                            ((x, x[:, :1], table), {}, "B x L"), ((x, None, table[0]), {}, "pairs x 2"),
                            ((x, None, table), dict(norm="batch"), "norm must"),
                            ((x, None, table), dict(w_k=w), "goes with k"),
                            ((x, x, table), dict(w_q=w, w_k=torch.ones(2, 8)), "both"),
                            ((x, None, table), dict(start=1 << 62), r"2\^62"), ((one(1, FAR, 2, 8), None, table), {}, r"2\^31")):
        with pytest.raises(ValueError, match=text):
            P.pam_head_norm_rotary_fwd(*args, **how)
        with pytest.raises(ValueError, match=text):
            P.pam_head_norm_rotary_bwd(*args, x, x, **how)
    c = torch.zeros(3, 2, 4, 8)
    for args, text in (((c, c), "device"), ((c[0], c), "pages"), ((c, c[:2]), "pages"), ((c.double(), c), "cache is"),
                       ((c[:, :, :, None].expand(3, 2, 4, 3, 8), c), "pages")):
        with pytest.raises(ValueError, match=text):
            P.PagedCache(*args)


def test_binding_refuses_what_does_not_fit_a_cache():
    """On a cache whose tensors are pretended to lie on the device."""
    cache = P.PagedCache.__new__(P.PagedCache)
    cache.k = cache.v = torch.zeros(3, 2, 4, 8, dtype=torch.bfloat16)
    cache.device, cache.maps, cache._sizes, cache._pool = 0, 1, (3, 4, 2, 8, 8, 1), [None] * 4
    t, n = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    k = torch.zeros(2, 5, 2, 8, dtype=torch.bfloat16)
    for bad in ((k[0], k), (k, k[:, :2]), (k[:, :, :1], k), (k[..., :4], k), (k[:, :, :, None], k)):
        with pytest.raises(ValueError, match="B x L"):
            P.pam_cache_write(cache, *bad, t, n)
    with pytest.raises(ValueError, match="B x L x H"):
        P.pam_paged_attn(k[0], cache, t, n)
    with pytest.raises(ValueError, match="B x L x H"):
        P.pam_paged_attn(k[..., :4], cache, t, n)
    with pytest.raises(ValueError, match="two maps"):
        P.pam_paged_attn(k, cache, t, n, lam=torch.zeros(2))
