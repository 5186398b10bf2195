"""Parity of the operators around an attention layer (through the C ABI) with
the 64-bit oracle (oracle/attn.py).

Bounds.  A result is compared value by value.  With u the unit roundoff of the
activations' type (2^-8 bf16, 2^-11 fp16, 2^-24 fp32: half a unit in the last
place, relative) and the oracle's magnitude of a result (the sum of the
absolute values of its terms), a kernel may be off by
  * u |result|: it is rounded once when it is stored;
  * for probabilities, score gradients and saved outputs, which are rounded to
    the activations' type before they meet the matrix units, u times the
    magnitude that they enter with;
  * 32-bit arithmetic: 2^-24 times the number of operations in a chain, times
    the magnitude.  A score of magnitude S is off by (d + 4) 2^-24 S and moves
    its probability by that factor; sums over n terms add n 2^-24 at the most.
"""
import numpy as np
import pytest

from helpers import log
from oracle import attn as A

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}  # below it a type has no relative precision


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_1907_00641_amd.binding as B

    B.lib()


def dt(name):
    import torch

    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def dev(a, name="f32"):
    """A numpy array on the GPU in the given type, and the values it holds there."""
    import torch

    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dt(name)).cuda()
    return t, host(t)


def host(t):
    return t.detach().double().cpu().numpy()


def check(name, got, want, bound):
    got = host(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert np.isfinite(got).all(), f"{name}: not finite"
    off = np.abs(got - want)
    worst = float((off / np.maximum(bound, 1e-300)).max()) if off.size else 0.0
    log(f"  {name}: largest error {off.max() if off.size else 0:.2e}, {worst:.2f} of its bound")
    assert worst <= 1.0, (name, worst)


# ---------------------------------------------------------------------------
# differential attention
# ---------------------------------------------------------------------------

class Case:
    def __init__(self, seed, B, lq, lk, H, hk, d, dv, t, causal=False, q_len=None, k_len=None, mask=None, scale=None,
                 spread=1.0):
        import torch

        rng = np.random.default_rng(seed)
        self.t, self.causal, self.scale = t, causal, d ** -0.5 if scale is None else scale
        self.q, self.qh = dev(spread * rng.standard_normal((B, lq, H, 2, d)), t)
        self.k, self.kh = dev(rng.standard_normal((B, lk, hk, 2, d)), t)
        self.v, self.vh = dev(rng.standard_normal((B, lk, hk, dv)), t)
        self.lam, self.lamh = dev(rng.uniform(0.2, 0.8, H), t)
        self.g, self.gh = dev(rng.standard_normal((B, lq, H, dv)), t)
        self.q_len, self.k_len = q_len, k_len
        self.mask = None if mask is None else rng.random((B, lk)) >= mask
        self.how = dict(scale=self.scale, causal=causal)
        for n, x in (("q_len", q_len), ("k_len", k_len)):
            if x is not None:
                self.how[n] = torch.tensor(x, dtype=torch.int32).cuda()
        if self.mask is not None:
            self.how["key_mask"] = torch.from_numpy(self.mask).cuda()
        self.see = A.visible(B, lq, lk, causal, q_len, k_len, self.mask)

    def run(self, **kw):
        import torch

        import paper_1907_00641_amd as P

        out, saved = P.pam_diff_attn_fwd(self.q, self.k, self.v, self.lam, save=True, **self.how, **kw)
        grads = P.pam_diff_attn_bwd(self.q, self.k, self.v, self.lam, saved, self.g, **self.how, **kw)
        torch.cuda.synchronize()
        return out, saved, grads

    def compare(self, out, saved=None, grads=None):
        r, a = A.attention(self.qh, self.kh, self.vh, self.lamh, self.scale, self.see,
                           self.gh if grads is not None else None)
        u, tiny = U[self.t], TINY[self.t]
        d, dv, lk, lq = self.qh.shape[-1], self.vh.shape[-1], self.kh.shape[1], self.qh.shape[1]
        S = A.score_size(self.qh, self.kh, self.scale)
        # a probability: its score, the exponential, the sum of its row
        e = 2.0 ** -24 * (2 * (d + 4) * S + 16 + lk)
        check("out", out, r["out"], u * np.abs(r["out"]) + (u + e) * a["out"] + tiny)
        if saved is not None:
            seen = np.isfinite(r["lse"])
            lse = host(saved[1])
            assert np.array_equal(np.isfinite(lse), seen), "rows that see something"
            off = np.abs(lse[seen] - r["lse"][seen])
            assert (off <= e + 2.0 ** -22 * np.abs(r["lse"][seen])).all(), off.max()
        if grads is None:
            return
        G = self.qh.shape[2] // self.kh.shape[2]
        ep = 2.0 ** -24 * (dv + 8)  # dp and D
        n = {"dq": lk, "dk": lq * G, "dv": lq * G}
        for i, name in enumerate(("dq", "dk")):
            A0, AD, AP = a[name]
            bound = u * np.abs(r[name]) + (u + e + n[name] * 2.0 ** -24) * A0 + (2 * u + 2 * e + ep) * AD + (e + ep) * AP
            check(name, grads[i], r[name], bound + tiny)
        check("dv", grads[2], r["dv"], u * np.abs(r["dv"]) + (u + e + n["dv"] * 2.0 ** -24) * a["dv"] + tiny)
        rows = self.qh.shape[0] * lq * 2.0 ** -24
        check("dlam", grads[3], r["dlam"], u * np.abs(r["dlam"]) + (e + ep + rows) * a["dlam"] + tiny)


SHAPES = [  # B, lq, lk, H, hk, d, dv
    (1, 1, 1, 1, 1, 16, 32),
    (2, 37, 53, 4, 2, 16, 32),
    (1, 64, 64, 2, 2, 32, 64),
    (2, 130, 97, 3, 1, 64, 128),
    (1, 70, 129, 2, 1, 128, 256),
    (1, 45, 66, 2, 2, 40, 80),
    (1, 33, 31, 3, 3, 5, 7),
    (1, 50, 70, 7, 1, 64, 64),
    (1, 40, 40, 2, 1, 24, 129),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_matches_oracle(shape, t, causal):
    log(f"[attn] {shape} {t} causal={causal}")
    c = Case(hash((shape, causal)) % 1000, *shape, t, causal=causal)
    c.compare(*c.run())


PART_SHAPES = [  # few tiles over a long axis, cut into parts that are joined
    (2, 300, 700, 4, 2, 32, 64),
    (1, 200, 600, 3, 1, 64, 128),
    (1, 150, 520, 2, 1, 128, 256),
    (1, 700, 300, 2, 2, 40, 80),
    (13, 140, 300, 20, 20, 8, 16),  # whole rounds of blocks, and then some
    (1, 140, 1100, 2, 2, 32, 64),
    (1, 300, 800, 4, 2, 64, 128),
    (2, 100, 1500, 3, 1, 40, 80),  # the kernel for few queries, cut
    (3, 250, 250, 14, 2, 64, 100),
    (20, 130, 130, 16, 16, 8, 16),  # causal: more than a round, the second blocks of the CUs in reverse
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", PART_SHAPES, ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_in_parts(shape, t, causal):
    log(f"[attn parts] {shape} {t} causal={causal}")
    c = Case(5, *shape, t, causal=causal)
    c.compare(*c.run())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_parts_that_see_nothing(t, causal):
    log(f"[attn empty parts] {t} causal={causal}")
    c = Case(6, 4, 300, 900, 4, 2, 32, 64, t, causal=causal, q_len=[0, 300, 130, 257], k_len=[900, 20, 0, 641], mask=0.5)
    c.compare(*c.run())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_len,k_len,mask", [([0, 70, 33], [0, 90, 91], None), ([70, 1, 64], [1, 0, 64], None),
                                              (None, [90, 32, 65], 0.5), (None, None, 0.9), (None, None, 1.0),
                                              ([-5, 1000, 3], [2, -1, 1000], None)],
                         ids=["ragged", "ones", "masked", "sparse", "all hidden", "clamped"])
def test_attention_lengths_and_masks(q_len, k_len, mask, causal, t):
    log(f"[attn masks] q_len={q_len} k_len={k_len} mask={mask} {t} causal={causal}")
    c = Case(77, 3, 70, 91, 4, 2, 32, 64, t, causal=causal, q_len=q_len, k_len=k_len, mask=mask)
    out, saved, grads = c.run()
    c.compare(out, saved, grads)
    nothing = ~c.see.any(axis=2)
    assert not host(out)[nothing].any() and not host(grads[0])[nothing].any()
    unseen = ~c.see.any(axis=1)
    assert not host(grads[1])[unseen].any() and not host(grads[2])[unseen].any()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lq", [70, 1])
def test_attention_hidden_places_may_hold_anything(t, lq):
    """NaN and infinities in keys and values past k_len or under the mask, in
    queries and upstream gradients past q_len: the same bits as with zeros there."""
    import torch

    c = Case(78, 2, lq, 150, 4, 2, 32, 64, t, k_len=[150, 101], q_len=[lq, max(lq - 9, 0)], mask=0.3)
    want = c.run()
    hide = torch.from_numpy(~c.mask).cuda()
    hide[1, 101:] = True
    c.k[hide], c.v[hide] = float("nan"), float("inf")
    c.k[1, 120:] = -float("inf")
    c.v[1, 130:] = float("nan")
    c.q[1, max(lq - 9, 0):], c.g[1, max(lq - 9, 0):] = float("nan"), float("inf")
    got = c.run()
    for a, b in zip([want[0], *want[1], *want[2]], [got[0], *got[1], *got[2]]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,dv", [(64, 128), (128, 256), (20, 40)])
@pytest.mark.parametrize("lq,causal", [(200, False), (200, True), (3, False)])
def test_attention_hidden_places_of_every_class(t, d, dv, lq, causal):
    """As above, for the other classes of head sizes, and over an axis that is cut into parts."""
    import torch

    c = Case(79, 2, lq, 330, 4, 2, d, dv, t, causal=causal, k_len=[330, 201], q_len=[lq, max(lq - 90, 1)], mask=0.3)
    want = c.run()
    hide = torch.from_numpy(~c.mask).cuda()
    hide[1, 201:] = True
    c.k[hide], c.v[hide] = float("nan"), float("inf")
    c.k[1, 220:] = -float("inf")
    c.v[1, 230:] = float("nan")
    c.q[1, max(lq - 90, 1):], c.g[1, max(lq - 90, 1):] = float("nan"), float("inf")
    got = c.run()
    for a, b in zip([want[0], *want[1], *want[2]], [got[0], *got[1], *got[2]]):
        assert torch.equal(a, b)
    c.compare(*want)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("d,dv", [(32, 64), (64, 128), (128, 256), (20, 36)])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_many_masked_keys(t, d, dv, causal):
    """Lengths, masks and NaN in hidden places where the keys are too many for the kernel for few queries."""
    import torch

    c = Case(80, 3, 150, 1100, 2, 1, d, dv, t, causal=causal, k_len=[1100, 0, 777], q_len=[150, 150, 41], mask=0.4)
    want = c.run()
    c.compare(*want)
    hide = torch.from_numpy(~c.mask).cuda()
    hide[2, 777:] = True
    c.k[hide], c.v[hide] = float("nan"), float("inf")
    c.k[1], c.v[1] = float("inf"), float("nan")
    c.q[2, 41:], c.g[2, 41:] = float("nan"), float("inf")
    got = c.run()
    for a, b in zip([want[0], *want[1], *want[2]], [got[0], *got[1], *got[2]]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_attention_many_keys_at_odd_strides(t):
    """Rows that start anywhere, NaN between them."""
    import torch

    c = Case(81, 1, 200, 1200, 3, 1, 40, 72, t, causal=True)
    for name in ("q", "k", "v"):
        x = getattr(c, name)
        wide = torch.full((*x.shape[:-1], x.shape[-1] + 5), float("nan"), dtype=x.dtype, device="cuda")
        wide[..., 3:-2] = x
        setattr(c, name, wide[..., 3:-2])
    c.compare(*c.run())


def test_attention_visible_nan_is_seen():
    """A NaN value that a row does see makes that row NaN and no other."""
    import torch

    import paper_1907_00641_amd as P

    c = Case(79, 2, 40, 80, 2, 1, 32, 64, "bf16", k_len=[80, 60])
    c.v[1, 59, 0, 3] = float("nan")
    out = P.pam_diff_attn_fwd(c.q, c.k, c.v, c.lam, **c.how)
    assert torch.isnan(out[1, :, :, 3]).all() and torch.isfinite(out[0]).all()
    assert torch.isfinite(out[1, :, :, 4:]).all()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_attention_large_scores(t):
    """Scores of some hundreds: one key takes nearly all of a row, exponentials of the others vanish."""
    c = Case(80, 1, 65, 130, 2, 1, 32, 64, t, spread=30.0)
    c.compare(*c.run())


@pytest.mark.parametrize("lq,lk,causal", [(1, 1, True), (1, 17, True), (1, 300, True), (1, 5000, False),
                                          (3, 2111, True), (2, 9001, True)])
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (14, 2)])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_decoding(lq, lk, causal, heads, t):
    import torch

    import paper_1907_00641_amd as P

    log(f"[decode] lq={lq} lk={lk} heads={heads} {t}")
    k_len = [lk, (lk * 2) // 3, 0]
    c = Case(lk, 3, lq, lk, *heads, 64, 128, t, causal=causal, k_len=k_len)
    out = P.pam_diff_attn_fwd(c.q, c.k, c.v, c.lam, **c.how)
    torch.cuda.synchronize()
    c.compare(out)
    out2, saved = P.pam_diff_attn_fwd(c.q, c.k, c.v, c.lam, save=True, **c.how)
    c.compare(out2, saved)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("off", [0, 1, 8])
def test_attention_strides(t, off):
    """q, k, v as parts of one packed projection and of a longer cache in another axis order, grad_out
    transposed, starts that are not 16-byte aligned; equal to the contiguous call."""
    import torch

    import paper_1907_00641_amd as P

    c = Case(81, 2, 50, 75, 4, 2, 32, 64, t, causal=True)
    want_out, saved, want = c.run()
    B, lq, H, _, d = c.q.shape
    wide = torch.full((B, lq, 2 * H * d + 24 + off), float("nan"), dtype=c.q.dtype, device="cuda")
    wide[:, :, off:off + 2 * H * d] = c.q.reshape(B, lq, -1)
    q = wide[:, :, off:off + 2 * H * d].view(B, lq, H, 2, d)
    cache = torch.full((2, B, 2, 90, 32 + off), float("nan"), dtype=c.k.dtype, device="cuda")  # map, seq, head, token
    cache[:, :, :, 10:85, :32] = c.k.permute(3, 0, 2, 1, 4)
    k = cache[:, :, :, 10:85, :32].permute(1, 3, 2, 0, 4)
    vbuf = torch.full((75, 2, B, 64 + 2 * off), float("nan"), dtype=c.v.dtype, device="cuda")
    vbuf[..., off:64 + off] = c.v.permute(1, 2, 0, 3)
    v = vbuf[..., off:64 + off].permute(2, 0, 1, 3)
    g = c.g.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
    out, sv = P.pam_diff_attn_fwd(q, k, v, c.lam, save=True, **c.how)
    grads = P.pam_diff_attn_bwd(q, k, v, c.lam, sv, g, **c.how)
    for a, b in zip((want_out, *saved, *want), (out, *sv, *grads)):
        assert torch.equal(a, b)


def test_attention_offsets_past_32_bits():
    """A cache whose tokens lie 2^25 elements apart (9 10^9 elements in all)."""
    import torch

    import paper_1907_00641_amd as P

    for lq in (40, 1):
        c = Case(82, 1, lq, 270, 2, 1, 32, 64, "bf16", causal=True)
        want = c.run()
        far = 1 << 25
        buf = torch.empty(270 * far, dtype=torch.bfloat16, device="cuda")
        k = buf.as_strided((1, 270, 1, 2, 32), (0, far, 0, 32, 1))
        v = buf.as_strided((1, 270, 1, 64), (0, far, 0, 1), 4096)
        k.copy_(c.k)
        v.copy_(c.v)
        out, saved = P.pam_diff_attn_fwd(c.q, k, v, c.lam, save=True, **c.how)
        grads = P.pam_diff_attn_bwd(c.q, k, v, c.lam, saved, c.g, **c.how)
        for a, b in zip((want[0], *want[2]), (out, *grads)):
            assert torch.equal(a, b)
        del buf, k, v


def test_attention_repeats_and_other_stream():
    """Two calls give the same bits, also on a stream of their own."""
    import torch

    c = Case(83, 2, 300, 500, 6, 2, 64, 128, "bf16", causal=True)
    first = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second, third = c.run(), c.run(stream=side)
    for a, b, d in zip(*[(x[0], *x[1], *x[2]) for x in (first, second, third)]):
        assert torch.equal(a, b) and torch.equal(a, d)


def test_operators_in_a_graph():
    """Captured once and replayed over new inputs, with eager work between the
    replays: every replay equals the eager calls."""
    import torch

    import paper_1907_00641_amd as P

    c = Case(84, 2, 96, 160, 4, 2, 32, 64, "bf16", causal=True, k_len=[160, 77])
    x = torch.randn(192, 128, device="cuda").bfloat16()
    z = c.v.new_empty(192, 128)
    w = torch.rand(128, device="cuda")

    def step():
        out, saved = P.pam_diff_attn_fwd(c.q, c.k, c.v, c.lam, save=True, **c.how)
        grads = P.pam_diff_attn_bwd(c.q, c.k, c.v, c.lam, saved, c.g, **c.how)
        one = P.pam_diff_attn_fwd(c.q[:, :1], c.k, c.v, c.lam, k_len=c.how["k_len"])
        z.copy_(out.reshape(192, 256)[:, :128])
        r, h = P.pam_norm_gate_fwd(x, z=z, w_post=w, w_pre=w, p=0.2, seed=5)
        g = P.pam_norm_gate_bwd(x, z=z, w_post=w, w_pre=w, p=0.2, seed=5, grad_r=r, grad_h=h)
        return [out, *grads, one, r, h, g["x"], g["z"], g["w_post"], P.pam_dropout(x, 0.5, 3)]

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for k in range(4):
        c.q.copy_(torch.randn_like(c.q, dtype=torch.float32))
        c.v.copy_(torch.randn_like(c.v, dtype=torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(held, want)):
            assert torch.equal(a, b), (k, i)


def test_attention_refuses_on_the_device_side():
    import torch

    import paper_1907_00641_amd as P

    c = Case(85, 2, 8, 8, 4, 2, 16, 32, "bf16")
    how = (c.q, c.k, c.v, c.lam)
    for bad in (dict(k_len=torch.zeros(2, dtype=torch.int64).cuda()), dict(k_len=torch.zeros(3, dtype=torch.int32).cuda()),
                dict(q_len=torch.zeros(2, dtype=torch.int32)), dict(key_mask=torch.ones(2, 8).cuda()),
                dict(key_mask=torch.ones(2, 9, dtype=torch.bool).cuda())):
        with pytest.raises(ValueError):
            P.pam_diff_attn_fwd(*how, **bad)
    with pytest.raises(ValueError):
        P.pam_diff_attn_fwd(c.q, c.k.float(), c.v, c.lam)
    with pytest.raises(ValueError):
        P.pam_diff_attn_fwd(c.q, c.k, c.v, c.lam.float())
    with pytest.raises(ValueError):
        P.pam_diff_attn_fwd(c.q.transpose(3, 4).contiguous().transpose(3, 4), c.k, c.v, c.lam)
    with pytest.raises(P.PamError):
        P.pam_diff_attn_fwd(*how, scale=-1.0)
    out, saved = P.pam_diff_attn_fwd(*how, save=True)
    with pytest.raises(ValueError):
        P.pam_diff_attn_bwd(*how, saved, c.g[:, :4])
    with pytest.raises(ValueError):
        P.pam_diff_attn_bwd(*how, (saved[0][0], saved[1]), c.g)


@pytest.mark.parametrize("lq,lk", [(0, 5), (5, 0), (0, 0)])
def test_attention_without_tokens(lq, lk):
    import torch

    c = Case(86, 2, lq, lk, 4, 2, 16, 32, "bf16")
    out, saved, (dq, dk, dv, dl) = c.run()
    assert out.shape == (2, lq, 4, 32) and not out.any() and not dq.any() and not dk.any() and not dv.any()
    assert torch.equal(dl, torch.zeros_like(dl))


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (128, 48), (80, 40), (6, 4), (20, 6), (40, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(t, d, rot, interleaved):
    import torch

    import paper_1907_00641_amd as P

    B, n, H, hk, entries = 2, 19, 6, 3, 50
    rng = np.random.default_rng(d + rot)
    freq, mag = P.pam_rotary_frequencies(rot, 10000.0, "yarn", 4.0, 512.0)
    table = P.pam_rotary_table(freq.cuda(), entries, magnitude=mag)
    ang = np.arange(entries)[:, None] * freq.numpy()
    tb = host(table)
    assert np.abs(tb[..., 0] - mag * np.cos(ang)).max() < 2.0 ** -23 and np.abs(tb[..., 1] - mag * np.sin(ang)).max() < 2.0 ** -23
    q, qh = dev(rng.standard_normal((B, n, H, d)), t)
    k, kh = dev(rng.standard_normal((B, n, hk, d)), t)
    pos = rng.integers(0, entries, (B, n)).astype(np.int32)
    for inverse in (False, True):
        for p in (torch.from_numpy(pos).cuda(), None):
            qo, ko = P.pam_rotary(q, k, table, pos=p, start=7, interleaved=interleaved, inverse=inverse)
            at = pos if p is not None else np.broadcast_to(7 + np.arange(n), (B, n))
            for name, y, x in (("q", qo, qh), ("k", ko, kh)):
                want = A.rotate(x, tb[at][..., 0], tb[at][..., 1], interleaved, inverse)
                big = A.rotate(np.abs(x), np.abs(tb[at][..., 0]), np.abs(tb[at][..., 1]), interleaved)
                size = np.abs(big) + 2 * np.abs(x).max()
                check(name, y, want, U[t] * np.abs(want) + 2.0 ** -22 * size + TINY[t])
                assert np.array_equal(host(y)[..., rot:], x[..., rot:])
    # a strided input, no k, in place
    wide = torch.full((B, n, H, d + 3), float("nan"), dtype=q.dtype, device="cuda")
    wide[..., :d] = q
    a, none = P.pam_rotary(wide[..., :d], None, table, start=3, interleaved=interleaved)
    b, _ = P.pam_rotary(q, None, table, start=3, interleaved=interleaved)
    assert none is None and torch.equal(a, b)
    P.pam_rotary(q, k, table, start=3, interleaved=interleaved, out=(q, k))
    assert torch.equal(q, b)


def test_rotary_table_of_voxels_and_far_positions():
    import torch

    import paper_1907_00641_amd as P

    rng = np.random.default_rng(3)
    freq = (10.0 ** -rng.uniform(0, 4, 12))
    coord = rng.uniform(-300000, 300000, (101, 3)).astype(np.float32)
    axis = np.repeat(np.arange(3, dtype=np.int32), 4)
    table = host(P.pam_rotary_table(torch.from_numpy(freq).cuda(), coord=torch.from_numpy(coord).cuda(),
                                    axis=torch.from_numpy(axis).cuda()))
    ang = coord.astype(np.float64)[:, axis] * freq
    assert np.abs(table[..., 0] - np.cos(ang)).max() < 2.0 ** -23 and np.abs(table[..., 1] - np.sin(ang)).max() < 2.0 ** -23


def test_rotary_outside_the_table_is_nan():
    import torch

    import paper_1907_00641_amd as P

    table = P.pam_rotary_table(P.pam_rotary_frequencies(8)[0].cuda(), 10)
    q = torch.randn(1, 4, 2, 16, device="cuda")
    pos = torch.tensor([[0, 10, -1, 9]], dtype=torch.int32).cuda()
    out, _ = P.pam_rotary(q, None, table, pos=pos)
    assert torch.isnan(out[0, 1:3, :, :8]).all() and torch.isfinite(out[0, [0, 3]]).all()
    assert torch.equal(out[..., 8:], q[..., 8:])
    out, _ = P.pam_rotary(q, None, table, start=8)
    assert torch.isfinite(out[0, :2]).all() and torch.isnan(out[0, 2:, :, :8]).all()


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 1000, 4099])
@pytest.mark.parametrize("p", [0.0, 0.25, 1.0])
def test_dropout(t, n, p):
    import torch

    import paper_1907_00641_amd as P

    x, xh = dev(np.random.default_rng(n).standard_normal(n + 1), t)
    seed, offset = 0x123456789ABCDEF, 0xFEDCBA987654321
    m = A.dropout_factors(n, p, seed, offset)
    for part, ph in ((x[:n], xh[:n]), (x[1:], xh[1:])):  # the second is not 16-byte aligned
        y = P.pam_dropout(part, p, seed, offset)
        got = host(y)
        assert np.array_equal(got == 0, (m == 0) | (ph == 0))
        check("y", y, ph * m, U[t] * np.abs(ph * m) * (1 + 2.0 ** -10) + 2.0 ** -23 * np.abs(ph * m) + TINY[t])
    y = P.pam_dropout(x[:n], p, seed, offset)
    xi = x[:n].clone()
    xi[torch.from_numpy(m == 0).cuda()] = float("nan")  # dropped whatever it holds
    assert torch.equal(P.pam_dropout(xi, p, seed, offset, out=xi), y)


def test_dropout_elements_past_32_bits():
    import torch

    import paper_1907_00641_amd as P

    n = (1 << 32) + 16
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    y = P.pam_dropout(x, 0.5, 77, 5, out=x)
    m = A.dropout_factors(4096, 0.5, 77, 5, first=n - 4096)
    assert np.array_equal(host(y[-4096:]), m)
    assert abs(float((y[:1 << 24] != 0).float().mean()) - 0.5) < 1e-3


# ---------------------------------------------------------------------------
# norms, gate, residual scale
# ---------------------------------------------------------------------------

NORM_SHAPES = [  # rows, channels, gate rows (0: none)
    (1, 1, 0), (5, 18, 0), (24, 64, 8), (12, 75, 4), (33, 128, 33), (40, 256, 1), (10, 512, 5), (6, 771, 3),
    (9, 1024, 0), (4, 2048, 2), (5, 4096, 0), (3, 8192, 3), (3, 8001, 1), (2500, 32, 2), (1500, 40, 1), (700, 16, 350),
    (300, 8192, 1), (520, 4099, 2), (1100, 700, 1), (900, 1600, 1),  # more gate rows than blocks
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("n,c,gate_rows", NORM_SHAPES, ids=str)
def test_norm_gate(n, c, gate_rows, norm, t):
    import paper_1907_00641_amd as P

    log(f"[norm] {n}x{c} gate rows {gate_rows} {norm} {t}")
    rng = np.random.default_rng(n * c)
    p, seed, offset = (0.25, 99, 1 << 40) if n * c < 60000 and n % 2 else (0.0, 0, 0)
    arr = {"x": 2 * rng.standard_normal((n, c)), "z": rng.standard_normal((n, c))}
    if gate_rows:
        arr["gate"] = rng.standard_normal((n // gate_rows, c))
    dr, drh = dev(rng.standard_normal((n, c)), t)
    dh, dhh = dev(rng.standard_normal((n, c)), t)
    T, H = {}, {}
    for k, v in arr.items():
        T[k], H[k] = dev(v, t)
    vecs = {k: m + 0.3 * rng.standard_normal(c) for k, m in (("w_post", 1), ("b_post", 0), ("scale", 0.5), ("w_pre", 1),
                                                             ("b_pre", 0))}
    if norm == "rms" and n % 2:
        del vecs["b_post"], vecs["b_pre"]
    for k, v in vecs.items():
        T[k], H[k] = dev(v)
    eps = 1e-5
    m = A.dropout_factors(n * c, p, seed, offset).reshape(n, c) if p else None
    full = {k: H.get(k) for k in ("x", "z", "w_post", "b_post", "gate", "scale", "w_pre", "b_pre")}
    res, mag = A.norm_gate(**full, layer=norm == "layer", eps=np.float32(eps).astype(float), m=m, grad_r=drh, grad_h=dhh)
    how = dict(norm=norm, eps=eps, p=p, seed=seed, offset=offset, **{k: v for k, v in T.items() if k != "x"})
    r, h = P.pam_norm_gate_fwd(T["x"], **how)
    grads = P.pam_norm_gate_bwd(T["x"], grad_r=dr, grad_h=dh, **how)
    u, e = U[t], 256 * 2.0 ** -24
    check("r", r, res["r"], u * np.abs(res["r"]) + e * mag["r"] + TINY[t])
    check("h", h, res["h"], u * np.abs(res["h"]) + e * mag["h"] + TINY[t])
    for k in T:
        vec = k in vecs
        bound = (0 if vec else u) * np.abs(res[k]) + (e + (n * 2.0 ** -24 if vec or k == "gate" else 0)) * mag[k]
        check("d" + k, grads[k], res[k], bound + (TINY[t] if not vec else 0))


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_norm_parts(t):
    """No block before, no norm after, no upstream gradient of r, strided rows, in place."""
    import torch

    import paper_1907_00641_amd as P

    n, c = 37, 96
    x, xh = dev(np.random.default_rng(1).standard_normal((n, c)), t)
    z, zh = dev(np.random.default_rng(2).standard_normal((n, c)), t)
    w, wh = dev(np.random.default_rng(3).standard_normal(c))
    g, gh = dev(np.random.default_rng(4).standard_normal((n, c)), t)
    u, e = U[t], 256 * 2.0 ** -24
    eps = float(np.float32(1e-6))

    def o(z=None, w_post=None, w_pre=None, **kw):
        return A.norm_gate(xh, z, w_post, None, None, None, w_pre, None, False, eps, None, **kw)

    r, h = P.pam_norm_gate_fwd(x, w_pre=w)
    res, mag = o(w_pre=wh, grad_h=gh)
    assert r is None
    check("h", h, res["h"], u * np.abs(res["h"]) + e * mag["h"] + TINY[t])
    grads = P.pam_norm_gate_bwd(x, w_pre=w, grad_r=None, grad_h=g)
    check("dx", grads["x"], res["x"], u * np.abs(res["x"]) + e * mag["x"] + TINY[t])
    check("dw", grads["w_pre"], res["w_pre"], (e + n * 2.0 ** -24) * mag["w_pre"])
    assert grads["z"] is None
    r, h = P.pam_norm_gate_fwd(x, z=z, w_post=w, next_norm=False)
    res, mag = o(z=zh, w_post=wh, grad_r=gh)
    assert h is None
    check("r", r, res["r"], u * np.abs(res["r"]) + e * mag["r"] + TINY[t])
    grads = P.pam_norm_gate_bwd(x, z=z, w_post=w, grad_r=g, grad_h=None)
    assert torch.equal(grads["x"], g)
    check("dz", grads["z"], res["z"], u * np.abs(res["z"]) + e * mag["z"] + TINY[t])
    check("dw", grads["w_post"], res["w_post"], (e + n * 2.0 ** -24) * mag["w_post"])
    for pad in (8, 3):
        xw = torch.full((n, c + pad), float("nan"), dtype=x.dtype, device="cuda")
        zw = torch.full((n, c + 2 * pad), float("nan"), dtype=x.dtype, device="cuda")
        xw[:, :c], zw[:, :c] = x, z
        r2, _ = P.pam_norm_gate_fwd(xw[:, :c], z=zw[:, :c], w_post=w, next_norm=False)
        if pad == 8:
            assert torch.equal(r, r2)
        else:  # other lanes hold the row: another order of its sum
            check("r", r2, res["r"], u * np.abs(res["r"]) + e * mag["r"] + TINY[t])
    empty = P.pam_norm_gate_bwd(x[:0], z=z[:0], w_post=w, grad_r=g[:0], grad_h=None)
    assert empty["x"].shape == (0, c) and not empty["w_post"].any()
    assert P.pam_norm_gate_fwd(x[:0], z=z[:0], w_pre=w)[1].shape == (0, c)


def test_norm_repeats():
    import torch

    import paper_1907_00641_amd as P

    x, z, g = (torch.randn(3000, 512, device="cuda").bfloat16() for _ in range(3))
    gate = torch.randn(3, 512, device="cuda").bfloat16()
    w = torch.rand(512, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b, d = (P.pam_norm_gate_bwd(x, z=z, w_post=w, gate=gate, w_pre=w, grad_r=g, grad_h=g, p=0.1, seed=4, stream=s)
               for s in (None, None, side))
    torch.cuda.synchronize()
    for k in a:
        assert a[k] is None or (torch.equal(a[k], b[k]) and torch.equal(a[k], d[k])), k
