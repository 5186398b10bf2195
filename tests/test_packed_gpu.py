"""Parity of attention over packed sequences and from a paged cache (through the C ABI) with the 64-bit oracle
(oracle/packed.py).

Bounds.  A result is compared value by value.  With u the unit roundoff of the activations' type (2^-8 bf16, 2^-11
fp16, 2^-24 fp32: half a unit in the last place, relative) and the oracle's magnitude of a result (the sum of the
absolute values of its terms), a kernel may be off by
  * u |result|: it is rounded once when it is stored;
  * for probabilities and score gradients, which are rounded to the activations' type before they meet the matrix
    units, u times the magnitude that they enter with; for 8-bit values that are scaled in fp16 another u;
  * 32-bit arithmetic: 2^-24 times the number of operations in a chain, times the magnitude.  A score of magnitude S
    is off by (d + 6) 2^-24 S and moves its probability by that factor; sums over n terms add n 2^-24 at the most.
"""
import numpy as np
import pytest

from helpers import log
from oracle import packed as O
from test_attn_gpu import TINY, U, _cuda, check, dev, dt, host  # noqa: F401

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def ints(x):
    import torch

    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def same(a, b):
    """Equal bits (NaN equal to NaN)."""
    import torch

    if a is None or b is None:
        return a is b
    if isinstance(a, (tuple, list)):
        return all(same(x, y) for x, y in zip(a, b))
    return a.shape == b.shape and bool(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)))


# ---------------------------------------------------------------------------
# attention over packed sequences
# ---------------------------------------------------------------------------

class Packed:
    def __init__(self, seed, lens, prefix, H, hk, d, dv, t, causal=True, before=0, behind=0, spread=1.0, k_lens=None):
        rng = np.random.default_rng(seed)
        k_lens = [n + prefix for n in lens] if k_lens is None else k_lens
        self.t, self.causal, self.scale = t, causal, d ** -0.5
        self.q_ends = [before + sum(lens[:b]) for b in range(len(lens) + 1)]
        self.k_ends = [before // 2 + sum(k_lens[:b]) for b in range(len(lens) + 1)]
        T, S = self.q_ends[-1] + behind, self.k_ends[-1] + behind
        self.q, self.qh = dev(spread * rng.standard_normal((T, H, d)), t)
        self.k, self.kh = dev(rng.standard_normal((S, hk, d)), t)
        self.v, self.vh = dev(rng.standard_normal((S, hk, dv)), t)
        self.g, self.gh = dev(rng.standard_normal((T, H, dv)), t)
        self.how = dict(scale=self.scale, causal=causal, q_start=ints(self.q_ends), k_start=ints(self.k_ends))

    def run(self, **kw):
        import torch

        import paper_1907_00641_amd as P

        out, saved = P.pam_attn_fwd(self.q, self.k, self.v, save=True, **self.how, **kw)
        grads = P.pam_attn_bwd(self.q, self.k, self.v, saved, self.g, **self.how, **kw)
        torch.cuda.synchronize()
        return (out, *grads), saved

    def compare(self, results, saved=None):
        r, a = O.packed(self.qh, self.kh, self.vh, self.scale, self.q_ends, self.k_ends, self.causal, self.gh)
        u, tiny = U[self.t], TINY[self.t]
        d, dv = self.qh.shape[-1], self.vh.shape[-1]
        H, hk = self.qh.shape[1], self.kh.shape[1]
        lens = np.diff(self.q_ends)
        lk, lq = int(np.diff(self.k_ends).max(initial=0)), int(lens.max(initial=0)) * (H // hk)
        S = self.scale * np.linalg.norm(self.qh, axis=-1).max(initial=0) * np.linalg.norm(self.kh, axis=-1).max(initial=0)
        e = E * (2 * (d + 6) * S + 16 + lk)  # a probability: its score, the exponential, the sum of its row
        check("out", results[0], r["out"], u * np.abs(r["out"]) + (u + e) * a["out"] + tiny)
        ep = E * (dv + 8)  # dp and D
        for name, got, n in (("dq", results[1], lk), ("dk", results[2], lq)):
            A0, AD, AP = a[name]
            check(name, got, r[name], u * np.abs(r[name]) + (u + e + n * E) * A0 + (2 * e + ep) * (AD + AP) + tiny)
        check("dv", results[3], r["dv"], u * np.abs(r["dv"]) + (u + e + lq * E) * a["dv"] + tiny)
        if saved is not None:
            inside = np.zeros(self.qh.shape[0], dtype=bool)
            inside[self.q_ends[0]:self.q_ends[-1]] = True
            lse, want = host(saved[1])[:, inside], r["lse"][:, inside]
            seen = np.isfinite(want)
            assert np.array_equal(np.isfinite(lse), seen)
            assert (np.abs(lse[seen] - want[seen]) <= e + 2.0 ** -22 * np.abs(want[seen])).all()


PACKED = [  # lens, prefix, H, hk, d, dv
    ([1], 0, 1, 1, 16, 16),
    ([1, 1, 1], 2, 2, 1, 64, 64),
    ([37, 1, 130, 64], 0, 4, 2, 40, 24),
    ([129, 0, 63], 5, 3, 1, 128, 128),
    ([31, 33], 0, 3, 3, 5, 7),
    ([200], 100, 7, 1, 64, 128),
    ([128, 256], 0, 2, 2, 80, 80),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", PACKED, ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_matches_oracle(shape, t, causal):
    log(f"[packed] {shape} {t} causal={causal}")
    c = Packed(len(str(shape)), *shape, t, causal)
    c.compare(*c.run())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("k_lens", [[0, 90, 64, 0], [90, 20, 1, 63], [10, 0, 0, 200]], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_more_queries_than_keys(k_lens, t, causal):
    """Causal rows that see nothing, and sequences without keys or without queries."""
    log(f"[packed] k_lens={k_lens} {t} causal={causal}")
    c = Packed(7, [70, 33, 0, 150], 0, 4, 2, 32, 48, t, causal, k_lens=k_lens)
    res, saved = c.run()
    c.compare(res, saved)
    nothing = ~np.isfinite(O.packed(c.qh, c.kh, c.vh, c.scale, c.q_ends, c.k_ends, causal)[0]["lse"]).T
    assert not host(res[0])[nothing].any() and not host(res[1])[nothing].any()


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("count", [64, 65, 150])
def test_attention_many_sequences(count, t, causal):
    """A sequence to a lane, and more than that; lengths of zero among them, tiles of several sequences."""
    log(f"[packed] {count} sequences {t} causal={causal}")
    rng = np.random.default_rng(count)
    lens = [int(x) for x in rng.choice([0, 1, 17, 64, 128, 129, 300], count)]
    c = Packed(8, lens, 3, 2, 1, 24, 24, t, causal)
    c.compare(*c.run())


PARTS = [([700], 0, 2, 1, 64, 64), ([300, 500], 300, 2, 1, 128, 128), ([40], 1100, 3, 1, 40, 24), ([1500, 10, 700], 0, 1, 1, 64, 32)]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", PARTS, ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_in_parts(shape, t, causal):
    """Few tiles over a long axis, cut into parts that are joined."""
    log(f"[packed parts] {shape} {t} causal={causal}")
    c = Packed(9, *shape, t, causal)
    c.compare(*c.run())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape,causal", [(([700, 650], 0, 44, 44, 16, 16), False), (([700, 650], 0, 44, 44, 16, 16), True),
                                          (([130] * 20, 0, 14, 7, 72, 72), False), (([130] * 20, 0, 14, 7, 72, 72), True),
                                          (([300] * 9, 7, 16, 4, 32, 32), True), (([300] * 9, 7, 16, 4, 32, 32), False),
                                          (([3100], 0, 8, 8, 16, 16), True), (([1500, 1300], 0, 8, 8, 72, 72), True),
                                          (([900, 40, 900], 0, 16, 8, 64, 64), False)], ids=str)
def test_attention_many_units(shape, causal, t):
    """About as many units as the card holds blocks, and more: whole rounds and a cut rest, one team of waves or two,
    the second blocks of the CUs in reverse, long causal walks in parts."""
    log(f"[packed units] {shape} {t} causal={causal}")
    c = Packed(22, *shape, t, causal)
    c.compare(*c.run())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d", [40, 64, 100])
@pytest.mark.parametrize("lens", [[70, 0, 129], [500], [140] * 40], ids=str)
def test_attention_rows_of_no_sequence(lens, d, t):
    """Before the first sequence and behind the last one: no part of anything, whatever they hold; their results 0."""
    import torch

    c = Packed(10, lens, 9, 4, 2, d, d, t, True, before=6, behind=70)
    want, _ = c.run()
    q0, q1, k0, k1 = c.q_ends[0], c.q_ends[-1], c.k_ends[0], c.k_ends[-1]
    for x, a, b in ((c.q, q0, q1), (c.g, q0, q1), (c.k, k0, k1), (c.v, k0, k1)):
        x[:a], x[b:] = float("nan"), float("inf")
    got, saved = c.run()
    assert same(got, want)
    assert not got[0][:q0].any() and not got[0][q1:].any() and not got[1][:q0].any() and not got[1][q1:].any()
    for x in got[2:]:
        assert not x[:k0].any() and not x[k1:].any()
    for x in (c.qh, c.gh):
        x[:q0], x[q1:] = 0, 0
    c.compare(got)
    assert torch.isfinite(got[0]).all()


def test_attention_starts_are_clamped():
    """Starts past the arrays, and below 0: the sequences that are left."""
    import paper_1907_00641_amd as P

    c = Packed(11, [60, 70], 0, 2, 1, 64, 64, "bf16")
    want = P.pam_attn_fwd(c.q, c.k, c.v, causal=True, q_start=ints([0, 60, 130]), k_start=ints([0, 60, 130]))
    got = P.pam_attn_fwd(c.q, c.k, c.v, causal=True, q_start=ints([-9, 60, 1000]), k_start=ints([-2 ** 31, 60, 2 ** 31 - 1]))
    assert same(got, want)
    # a sequence that ends before it starts is empty
    got = P.pam_attn_fwd(c.q, c.k, c.v, causal=True, q_start=ints([60, 0, 0]), k_start=ints([60, 0, 0]))
    assert got.shape == want.shape


def test_attention_without_starts_is_one_sequence():
    import paper_1907_00641_amd as P

    c = Packed(12, [300], 0, 4, 2, 64, 64, "bf16")
    want, saved = P.pam_attn_fwd(c.q, c.k, c.v, causal=True, save=True, q_start=ints([0, 300]), k_start=ints([0, 300]))
    got, saved2 = P.pam_attn_fwd(c.q, c.k, c.v, causal=True, save=True)
    assert same((got, *saved2), (want, *saved))
    assert same(P.pam_attn_bwd(c.q, c.k, c.v, saved, c.g, causal=True),
                P.pam_attn_bwd(c.q, c.k, c.v, saved, c.g, causal=True, q_start=ints([0, 300]), k_start=ints([0, 300])))


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_attention_is_each_sequence_alone(t):
    """The same rows, packed with others or alone: equal to rounding's order (the parts differ), and within bounds."""
    import paper_1907_00641_amd as P

    c = Packed(13, [77, 140, 5], 0, 2, 2, 48, 48, t)
    res, _ = c.run()
    for b in range(3):
        x, y = slice(c.q_ends[b], c.q_ends[b + 1]), slice(c.k_ends[b], c.k_ends[b + 1])
        one = P.pam_attn_fwd(c.q[x], c.k[y], c.v[y], causal=True, scale=c.scale)
        off = np.abs(host(one) - host(res[0][x])).max()
        assert off <= 2 * U[t] * (np.abs(host(one)).max() + np.abs(c.vh).max()) + 1e-5, (b, off)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("off", [1, 8])
def test_attention_strides(t, off):
    """q, k and v as parts of one projection, the heads outside, starts that are not 16-byte aligned, NaN between."""
    import torch

    import paper_1907_00641_amd as P

    c = Packed(14, [90, 40], 0, 4, 2, 40, 40, t)
    want, _ = c.run()
    T, H, d = c.q.shape
    both = torch.full((T, 3 * H * d + off), float("nan"), dtype=c.q.dtype, device="cuda")
    q = both[:, off:off + H * d].view(T, H, d)
    q.copy_(c.q)
    k = both[:, off + H * d:off + H * d + 2 * d].view(T, 2, d)
    k.copy_(c.k)
    v = torch.full((2, T, d + 3), float("nan"), dtype=c.v.dtype, device="cuda")[:, :, :d].transpose(0, 1)
    v.copy_(c.v)
    g = torch.empty(H, T, d, dtype=c.q.dtype, device="cuda").transpose(0, 1)
    g.copy_(c.g)
    out, saved = P.pam_attn_fwd(q, k, v, save=True, **c.how)
    grads = P.pam_attn_bwd(q, k, v, saved, g, **c.how)
    c.compare((out, *grads), saved)
    # backwards in memory, and a key that every head shares by a stride of 0
    flip = Packed(14, [90, 40], 0, 4, 2, 40, 40, t)
    back = torch.empty_like(flip.q)
    back.copy_(flip.q.flip(0))
    shared = flip.k[:, :1].expand(-1, 2, -1)
    got = P.pam_attn_fwd(back.flip(0).as_strided(flip.q.shape, flip.q.stride()), shared, flip.v, **flip.how)
    want = P.pam_attn_fwd(flip.q, shared.contiguous(), flip.v, **flip.how)
    assert np.abs(host(got) - host(want)).max() <= 4 * U[t] * (1 + np.abs(host(want)).max())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_attention_large_scores(t):
    """Scores of some hundreds: one key takes nearly all of a row."""
    c = Packed(15, [65, 130], 0, 2, 1, 32, 64, t, spread=30.0)
    c.compare(*c.run())


def test_attention_common_part_of_values():
    """Values around 4 times their deviation: the difference of dp and D is far smaller than either."""
    import torch

    c = Packed(16, [300], 0, 2, 1, 64, 64, "bf16")
    c.v += 4.0
    c.vh = host(c.v)
    c.compare(*c.run())
    r, _ = O.packed(c.qh, c.kh, c.vh, c.scale, c.q_ends, c.k_ends, True, c.gh)
    (_, dq, _, _), _ = c.run()
    assert np.linalg.norm(host(dq) - r["dq"]) < 0.005 * np.linalg.norm(r["dq"])
    assert torch.isfinite(dq).all()


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("lens", [[130], [130] * 70], ids=["few units", "many units"])
def test_attention_small_and_large_gradients(t, lens):
    """Upstream gradients of 1e-6 and, in bf16, 1e20."""
    import torch

    for size in (1e-6, 1e3) + ((1e20,) if t == "bf16" else ()):
        c = Packed(17, lens, 20, 2, 1, 64, 64, t)
        want, saved = c.run()
        g = (c.g.float() * size).to(c.g.dtype)
        c.g, c.gh = g, host(g)
        (_, *grads), _ = c.run()
        r, _ = O.packed(c.qh, c.kh, c.vh, c.scale, c.q_ends, c.k_ends, True, c.gh)
        for name, x in zip(("dq", "dk", "dv"), grads):
            assert torch.isfinite(x).all()
            off = np.abs(host(x) - r[name]).max()
            assert off <= 8 * U[t] * np.abs(r[name]).max() + 2 * TINY[t], (name, size, off)


def test_attention_gradients_against_differences():
    """fp32: sum(g out) along a direction, over 2 e.  The sum of 10^4 products of magnitude 1 in 64 bits from values that
    are off by 1e-6 at random is off by 1e-4; over 2 e = 0.04 that is 3e-3, of derivatives of some tens; the third
    derivative takes e^2 / 6 = 7e-5 of some hundreds."""
    import paper_1907_00641_amd as P

    c = Packed(18, [60, 97], 11, 4, 2, 24, 24, "f32")
    (_, *grads), _ = c.run()
    rng = np.random.default_rng(3)
    for name, g in zip("qkv", grads):
        x = getattr(c, name)
        step, _ = dev(rng.standard_normal(x.shape) * np.sign(host(g)))
        step = step.abs() * g.sign()
        keep, e, f = x.clone(), 0.02, []
        for s in (e, -e):
            x.copy_(keep + s * step)
            f.append((host(P.pam_attn_fwd(c.q, c.k, c.v, **c.how)) * c.gh).sum())
        x.copy_(keep)
        got, want = (f[0] - f[1]) / (2 * e), (host(g) * host(step)).sum()
        log(f"  {name}: {want:.4f} by the formula, {got:.4f} by differences")
        assert abs(got - want) <= 5e-3 * abs(want) + 0.1


def test_attention_repeats_and_streams():
    """Equal bits on repetition, on another stream, and where memory is handed out again at once."""
    import torch

    c = Packed(19, [700, 50, 333], 0, 4, 2, 64, 64, "bf16")
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = c.run(stream=side)
        side.synchronize()
        assert same(got, want)
        assert same(c.run(), want)


@pytest.mark.parametrize("lens", [[700, 50], [64, 64, 64], [400] * 60], ids=str)
def test_attention_in_a_graph(lens):
    """Forward and backward captured, replayed with eager calls between, and with other lengths in the same starts."""
    import torch

    c = Packed(20, lens, 0, 2, 1, 64, 64, "bf16")
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.run()
    torch.cuda.current_stream().wait_stream(side)
    import paper_1907_00641_amd as P

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, saved = P.pam_attn_fwd(c.q, c.k, c.v, save=True, **c.how)
        grads = P.pam_attn_bwd(c.q, c.k, c.v, saved, c.g, **c.how)
    for ends in (c.q_ends, [0] + [n // 2 for n in c.q_ends[1:]], c.q_ends):
        c.how["q_start"].copy_(ints(ends))
        c.how["k_start"].copy_(ints(ends))
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            eager = c.run()
            assert same((out, *grads), eager[0])
    assert same(eager[0], want[0])


def test_attention_far_offsets():
    """Rows whose offsets pass 2^32 bytes and 2^31 elements, read wide and element by element."""
    import torch

    import paper_1907_00641_amd as P

    for stride in (1 << 23, (1 << 23) + 3):
        n = 300
        pool = torch.empty(n * stride + 256, dtype=torch.bfloat16, device="cuda")
        c = Packed(21, [n], 0, 1, 1, 64, 64, "bf16")
        q, k, v = (pool[at:].as_strided((n, 1, 64), (stride, 64, 1)) for at in (0, 64, 128))
        for x, y in ((q, c.q), (k, c.k), (v, c.v)):
            x.copy_(y)
        c.compare(*(lambda o: ((o[0], *P.pam_attn_bwd(q, k, v, o[1], c.g, **c.how)), o[1]))(
            P.pam_attn_fwd(q, k, v, save=True, **c.how)))
        del pool, q, k, v
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# norms of heads, rotary positions
# ---------------------------------------------------------------------------

class Norm:
    def __init__(self, seed, B, n, H, hk, d, pairs, t, layer=False, per_head=False, interleaved=False, eps=1e-6,
                 weights=True, entries=None):
        import torch

        rng = np.random.default_rng(seed)
        self.t, self.layer, self.interleaved, self.eps = t, layer, interleaved, eps
        self.q, self.qh = dev(2 * rng.standard_normal((B, n, H, d)) + 0.5, t)
        self.k, self.kh = dev(2 * rng.standard_normal((B, n, hk, d)) - 0.5, t) if hk else (None, None)
        self.gq, self.gqh = dev(rng.standard_normal((B, n, H, d)), t)
        self.gk, self.gkh = dev(rng.standard_normal((B, n, hk, d)), t) if hk else (None, None)
        self.wq, self.wqh = dev(1 + 0.3 * rng.standard_normal((H, d) if per_head else d))
        self.wk, self.wkh = dev(1 + 0.3 * rng.standard_normal((hk, d) if per_head else d)) if hk else (None, None)
        if not weights:
            self.wq = self.wk = None
            self.wqh = self.wkh = np.ones(d)
        entries = n + 3 if entries is None else entries
        self.table, th = dev(rng.standard_normal((entries, pairs, 2)))
        self.pos = rng.integers(0, entries, (B, n))
        self.cos, self.sin = th[self.pos][..., 0], th[self.pos][..., 1]
        self.how = dict(w_q=self.wq, w_k=self.wk, norm="layer" if layer else "rms", eps=eps, interleaved=interleaved,
                        pos=torch.from_numpy(self.pos).to(torch.int32).cuda())

    def run(self, **kw):
        import torch

        import paper_1907_00641_amd as P

        y = P.pam_head_norm_rotary_fwd(self.q, self.k, self.table, **self.how, **kw)
        g = P.pam_head_norm_rotary_bwd(self.q, self.k, self.table, self.gq, self.gk, **self.how, **kw)
        torch.cuda.synchronize()
        return (*y, g["q"], g["k"], g["w_q"], g["w_k"])

    def compare(self, res):
        u, tiny, d = U[self.t], TINY[self.t], self.qh.shape[-1]
        for i, (x, w, g) in enumerate(((self.qh, self.wqh, self.gqh), (self.kh, self.wkh, self.gkh))):
            if x is None:
                continue
            r, a = O.head_norm(x, w, self.cos, self.sin, self.layer, self.eps, self.interleaved, g)
            name = "qk"[i]
            check(f"{name}'", res[i], r["y"], u * np.abs(r["y"]) + (2 * d + 24) * E * a["y"] + tiny)
            check(f"d{name}", res[2 + i], r["dx"], u * np.abs(r["dx"]) + (4 * d + 48) * E * a["dx"] + tiny)
            if res[4 + i] is not None:
                rows = x.shape[0] * x.shape[1] * x.shape[2]
                check(f"dw_{name}", res[4 + i], r["dw"], (2 * d + 24 + rows) * E * a["dw"])


NORMS = [  # B, n, H, hk, d, pairs
    (1, 1, 1, 0, 2, 1), (1, 1, 1, 1, 64, 32), (2, 5, 3, 1, 128, 64), (1, 9, 4, 4, 80, 20), (2, 3, 5, 2, 40, 12),
    (1, 7, 2, 1, 33, 8), (1, 4, 2, 2, 512, 256), (1, 3, 2, 1, 511, 1), (1, 6, 12, 3, 256, 64), (2, 2, 1, 0, 7, 3),
    (1, 5, 2, 1, 24, 4), (1, 300, 6, 2, 32, 16),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", NORMS, ids=str)
@pytest.mark.parametrize("layer,per_head,interleaved", [(False, False, False), (True, True, True), (False, True, False),
                                                        (True, False, False), (False, False, True)])
def test_head_norm_matches_oracle(shape, t, layer, per_head, interleaved):
    log(f"[head norm] {shape} {t} layer={layer} per_head={per_head} interleaved={interleaved}")
    c = Norm(31, *shape, t, layer, per_head, interleaved)
    c.compare(c.run())


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("per_head", [False, True])
def test_head_norm_many_rows(t, per_head):
    """More rows than the backward pass's blocks take in one turn, over a number of heads that no block holds."""
    c = Norm(32, 2, 900, 7, 3, 64, 32, t, per_head=per_head)
    c.compare(c.run())
    many = Norm(33, 1, 3, 1500, 700, 16, 8, t, per_head=per_head)  # more heads than blocks
    many.compare(many.run())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_head_norm_without_weights_positions_by_start(t):
    import torch

    import paper_1907_00641_amd as P

    c = Norm(34, 2, 6, 4, 2, 64, 32, t, weights=False, entries=20)
    c.how.pop("pos")
    c.how["start"] = 9
    table = host(c.table)
    c.cos, c.sin = (np.broadcast_to(table[9:15, :, i], (2, 6, 32)) for i in (0, 1))
    res = c.run()
    assert res[4] is None and res[5] is None
    c.compare(res)
    # the same as the two operators behind each other, but for the rounding between
    q2, k2 = P.pam_rotary(c.q, c.k, c.table, start=9)
    want = host(q2) / np.sqrt((c.qh ** 2).mean(-1, keepdims=True) + c.eps)
    bound = U[t] * (2 * np.abs(want) + 2 * np.abs(table).max() * 6) + 1e-5
    assert (np.abs(host(res[0]) - want) <= bound).all()
    assert torch.isfinite(res[0]).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_norm_positions_outside_the_table(t, interleaved):
    """NaN in the turned channels of that token, and no other; the copied channels stay."""
    import torch

    c = Norm(35, 2, 5, 3, 1, 48, 16, t, interleaved=interleaved)
    want = c.run()
    c.how["pos"][1, 2], c.how["pos"][0, 0] = -1, c.table.shape[0]
    got = c.run()
    out = torch.zeros(2, 5, dtype=torch.bool, device="cuda")
    out[1, 2] = out[0, 0] = True
    for i in (0, 1):
        assert torch.isnan(got[i][out][..., :32]).all()
        assert same(got[i][out][..., 32:], want[i][out][..., 32:]) and same(got[i][~out], want[i][~out])
        assert same(got[2 + i][~out], want[2 + i][~out]) and torch.isnan(got[2 + i][out][..., :32]).all()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,pairs", [(64, 32), (80, 20), (33, 8)])
def test_head_norm_strides_and_in_place(t, d, pairs):
    import torch

    import paper_1907_00641_amd as P

    c = Norm(36, 2, 7, 4, 2, d, pairs, t)
    want = c.run()
    both = torch.full((2, 7, 6 * d + 5), float("nan"), dtype=c.q.dtype, device="cuda")
    q, k = both[:, :, 1:1 + 4 * d].view(2, 7, 4, d), both[:, :, 1 + 4 * d:1 + 6 * d].view(2, 7, 2, d)
    q.copy_(c.q)
    k.copy_(c.k)
    y = P.pam_head_norm_rotary_fwd(q, k, c.table, **c.how)
    c2 = Norm(36, 2, 7, 4, 2, d, pairs, t)
    c2.q, c2.k = q, k
    c2.compare(c2.run())
    qt = torch.empty(2, 4, 7, d, dtype=c.q.dtype, device="cuda").transpose(1, 2)
    qt.copy_(c.q)
    y2 = P.pam_head_norm_rotary_fwd(qt, c.k, c.table, **c.how)
    assert same(y2, want[:2])
    assert np.abs(host(y[0]) - host(want[0])).max() <= 2 * U[t] * np.abs(host(want[0])).max()
    a, b = c.q.clone(), c.k.clone()
    got = P.pam_head_norm_rotary_fwd(a, b, c.table, out=(a, b), **c.how)
    assert got[0] is a and same((a, b), want[:2])


def test_head_norm_gradients_against_differences():
    """fp32; the sum of 10^3 products in 64 bits of values off by 1e-6 of 5: 2e-4, over 2 e = 0.02: 1e-2."""
    import paper_1907_00641_amd as P

    for layer in (False, True):
        c = Norm(37, 1, 6, 4, 2, 24, 8, "f32", layer=layer)
        res = c.run()
        rng = np.random.default_rng(4)
        for x, g in ((c.q, res[2]), (c.k, res[3]), (c.wq, res[4]), (c.wk, res[5])):
            step = (dev(rng.standard_normal(x.shape))[0].abs() * g.sign()).contiguous()
            keep, e, f = x.clone(), 0.01, []
            for s in (e, -e):
                x.copy_(keep + s * step)
                y = P.pam_head_norm_rotary_fwd(c.q, c.k, c.table, **c.how)
                f.append((host(y[0]) * c.gqh).sum() + (host(y[1]) * c.gkh).sum())
            x.copy_(keep)
            got, want = (f[0] - f[1]) / (2 * e), (host(g) * host(step)).sum()
            log(f"  layer={layer}: {want:.4f} by the formula, {got:.4f} by differences")
            assert abs(got - want) <= 5e-3 * abs(want) + 0.05


def test_head_norm_repeats_streams_graph():
    import torch

    import paper_1907_00641_amd as P

    c = Norm(38, 2, 500, 8, 2, 64, 32, "bf16")
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(stream=side)
    side.synchronize()
    assert same(got, want) and same(c.run(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.pam_head_norm_rotary_fwd(c.q, c.k, c.table, **c.how)
        g = P.pam_head_norm_rotary_bwd(c.q, c.k, c.table, c.gq, c.gk, **c.how)
    for scale in (1.0, 0.5, 1.0):
        c.gq.copy_(torch.from_numpy(c.gqh * scale).to(c.gq.dtype))
        graph.replay()
        torch.cuda.synchronize()
        assert same((*y, g["q"], g["k"], g["w_q"], g["w_k"]), c.run())


def test_head_norm_zero_rows():
    """A row of zeros is 0 / sqrt(eps); without rows the weights' gradients are 0."""
    import torch

    import paper_1907_00641_amd as P

    c = Norm(39, 1, 4, 2, 1, 64, 32, "f32")
    c.q[0, 1], c.qh[0, 1] = 0, 0
    c.compare(c.run())
    q = c.q[:, :0].contiguous()
    g = P.pam_head_norm_rotary_bwd(q, None, c.table, q, None, w_q=c.wq)
    assert g["q"].shape == q.shape and not g["w_q"].any() and torch.isfinite(g["w_q"]).all()


# ---------------------------------------------------------------------------
# the paged cache
# ---------------------------------------------------------------------------

def store_type(name):
    import torch

    return {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}.get(name) or dt(name)


def numbers(t):
    """Stored numbers on the host, in 64 bits."""
    return t.float().cpu().double().numpy()


class Cache:
    """A pool with pages dealt out at random; one page that is no sequence's."""

    def __init__(self, seed, B, total, page, hk, d, dv, t, store, maps=1, k_len=None):
        import torch

        import paper_1907_00641_amd as P

        rng = np.random.default_rng(seed)
        per = -(-total // page)
        self.pages, self.page, self.maps, self.t, self.store, self.total = B * per + 1, page, maps, t, store, total
        self.hk, self.d, self.dv = hk, d, dv
        self.table_h = rng.permutation(self.pages)[:B * per].reshape(B, per)
        self.table = ints(self.table_h)
        self.k_len_h = np.full(B, total) if k_len is None else np.asarray(k_len)
        self.k_len = ints(self.k_len_h)
        lead = (self.pages, hk, page)
        self.cache = P.PagedCache.empty(self.pages, page, hk, d, dv, maps=maps, dtype=store_type(store))
        self.fill(rng.standard_normal((*lead, maps * d)), rng.standard_normal((*lead, dv)))
        torch.cuda.synchronize()

    def fill(self, k, v):
        """Sets the whole pool; kn, vn are the values that it stands for."""
        import torch

        lead = k.shape[:3]
        k = k.reshape(*lead, self.maps, self.d)
        res = []
        for x, to, sc in ((k, self.cache.k, self.cache.k_scale), (v, self.cache.v, self.cache.v_scale)):
            if sc is None:
                t, y = dev(x, self.t)
                to.copy_(t.view_as(to))
                res.append(y)
                continue
            y, s = O.stored(np.asarray(x, dtype=np.float32), self.store)
            num = torch.from_numpy(y.astype(np.float32)).cuda().to(to.dtype)
            to.view(torch.uint8).copy_(num.reshape(to.shape).view(torch.uint8))
            sc.copy_(torch.from_numpy(s).cuda().view_as(sc))
            res.append(y * s.astype(np.float64)[..., None])
        self.kn, self.vn = res

    def gathered(self, length):
        k, live = O.gathered(self.kn, self.table_h, self.page, self.k_len_h, length)
        v, _ = O.gathered(self.vn, self.table_h, self.page, self.k_len_h, length)
        return k, v, live


STORES = ["same", "e4m3", "int8"]


def stored_as(t, store):
    return t if store == "same" else store


CACHES = [  # B, old, new, page, hk, d, dv, maps
    (1, 0, 1, 1, 1, 16, 16, 1), (2, 19, 1, 16, 2, 64, 64, 1), (3, 0, 37, 5, 2, 40, 24, 1), (2, 11, 9, 24, 1, 128, 128, 1),
    (1, 30, 3, 8, 3, 20, 40, 2), (2, 5, 20, 16, 2, 64, 128, 2), (1, 3, 4, 4, 1, 7, 5, 1), (1, 2, 6, 16, 1, 256, 256, 1),
    (1, 40, 8, 32, 2, 128, 256, 2),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("shape", CACHES, ids=str)
@pytest.mark.parametrize("how", ["padded", "ragged", "packed"])
def test_cache_write_and_read(shape, store, t, how):
    """The pool's every number and scale: new ones as the oracle stores them, all others as they were.  Read back, the
    product of number and scale (24 bits) rounded to the type."""
    import torch

    import paper_1907_00641_amd as P

    B, old, new, page, hk, d, dv, maps = shape
    log(f"[cache] {shape} {store} {t} {how}")
    store = stored_as(t, store)
    rng = np.random.default_rng(41)
    new_len = np.full(B, new)
    if how != "padded":
        new_len = rng.integers(0, new + 1, B)
    k_len = np.array([old + n if b % 2 == 0 else max(old - 2 * b, 0) + n for b, n in enumerate(new_len)])
    c = Cache(40, B, old + new, page, hk, d, dv, t, store, maps, k_len)
    size = np.exp2(rng.uniform(-3, 3, (B, new, hk, 1, 1)))
    k, kh = dev(rng.standard_normal((B, new, hk, maps, d)) * size, t)
    v, vh = dev(rng.standard_normal((B, new, hk, dv)) * size[..., 0], t)
    k[0, 0, 0], kh[0, 0, 0] = 0, 0
    before = [None if x is None else x.clone() for x in (c.cache.k, c.cache.v, c.cache.k_scale, c.cache.v_scale)]
    kt = k if maps == 2 else k[:, :, :, 0]
    if how == "packed":
        rows = [slice(0, n) for n in new_len]
        pk, pv = torch.cat([kt[b, r] for b, r in enumerate(rows)]), torch.cat([v[b, r] for b, r in enumerate(rows)])
        starts = np.concatenate([[0], np.cumsum(new_len)])
        pad = torch.full_like(pk[:1], float("nan")) if len(pk) else pk  # rows of no sequence
        P.pam_cache_write(c.cache, torch.cat([pk, pad]), torch.cat([pv, torch.zeros_like(v[0, :len(pad)])]), c.table,
                          c.k_len, starts=ints(starts))
    else:
        if how == "ragged":
            for b, n in enumerate(new_len):  # rows that are not new
                kt[b, n:], v[b, n:] = float("nan"), float("inf")
        P.pam_cache_write(c.cache, kt, v, c.table, c.k_len, new_len=None if how == "padded" else ints(new_len))
    torch.cuda.synchronize()
    # the expected pool
    touched = np.zeros((c.pages, hk, page), dtype=bool)
    for name, x, pool, scale, was, was_scale, values in (
            ("k", kh, c.cache.k, c.cache.k_scale, before[0], before[2], c.kn),
            ("v", vh[:, :, :, None], c.cache.v, c.cache.v_scale, before[1], before[3], c.vn[:, :, :, None])):
        want = numbers(was).reshape(values.shape)
        want_scale = None if scale is None else host(was_scale).reshape(values.shape[:-1])
        for b, n in enumerate(new_len):
            for i in range(n):
                p = k_len[b] - n + i
                if p < 0:
                    continue
                at = (c.table_h[b, p // page], slice(None), p % page)
                touched[at] = True
                if scale is None:
                    want[at] = values[at] = x[b, i]
                else:
                    y, s = O.stored(x[b, i], store)
                    want[at], want_scale[at] = y, s
                    values[at] = y * s.astype(np.float64)[..., None]
        assert np.array_equal(numbers(pool).reshape(want.shape), want), name
        if scale is not None:
            assert np.array_equal(host(scale).reshape(want_scale.shape), want_scale), name
    assert touched.any() or not new_len.any()
    length = old + new
    gk, gv = P.pam_cache_read(c.cache, c.table, c.k_len, length, dtype=dt(t))
    wk, wv, _ = c.gathered(length)
    for name, got, want in (("k", gk, wk.reshape(gk.shape)), ("v", gv, wv)):
        check(name, got, want, (U[t] + (0 if store == t else E)) * np.abs(want) + (0 if store == t else TINY[t]))


def test_cache_pages_that_are_not_there():
    """Negative and too large page numbers: nothing written, zeros read, no query sees them; lengths past the table."""
    import torch

    import paper_1907_00641_amd as P

    c = Cache(42, 2, 40, 8, 2, 64, 64, "bf16", "int8", k_len=[40, 1000])
    c.table[0, 1], c.table[1, 4], c.table_h[0, 1], c.table_h[1, 4] = -1, c.pages, -1, -1
    c.k_len_h = np.array([40, 40])
    before = c.cache.k.clone(), c.cache.v.clone()
    new = torch.ones(2, 40, 2, 64, dtype=torch.bfloat16, device="cuda")
    P.pam_cache_write(c.cache, new, new, c.table, ints([40, -3]))
    at = torch.ones(c.pages, dtype=torch.bool)
    at[[x for x in c.table_h[0] if x >= 0]] = False
    assert same(c.cache.k[at], before[0][at]) and same(c.cache.v[at], before[1][at])
    assert (c.cache.k[~at] == 127).all()
    c.cache.k.copy_(before[0])
    c.cache.v.copy_(before[1])
    c2 = Cache(42, 2, 40, 8, 2, 64, 64, "bf16", "int8", k_len=[40, 40])
    c2.table, c2.table_h, c2.k_len = c.table, c.table_h, c.k_len
    gk, gv = P.pam_cache_read(c2.cache, c2.table, c2.k_len, 45, dtype=torch.bfloat16)
    assert not gk[0, 8:16].any() and not gk[1, 32:].any() and not gv[:, 40:].any()
    q, qh = dev(np.random.default_rng(1).standard_normal((2, 2, 4, 64)), "bf16")
    Paged.compare_with(c2, q, qh, None, None, None, P.pam_paged_attn(q, c2.cache, c2.table, c2.k_len))


@pytest.mark.parametrize("store", ["e4m3", "int8"])
def test_cache_rows_that_are_not_finite(store):
    """The whole row is NaN, and no other; a row of zeros and one of the smallest numbers."""
    import torch

    import paper_1907_00641_amd as P

    c = Cache(43, 1, 16, 16, 2, 64, 64, "f32", store)
    k = torch.randn(1, 16, 2, 64, device="cuda")
    k[0, 3, 1, 5], k[0, 7, 0, 63], k[0, 9], k[0, 11, 0] = float("nan"), -float("inf"), 0.0, 1e-42
    P.pam_cache_write(c.cache, k, k, c.table, c.k_len)
    got, _ = P.pam_cache_read(c.cache, c.table, c.k_len, 16, dtype=torch.float32)
    bad = torch.zeros(16, 2, dtype=torch.bool, device="cuda")
    bad[3, 1] = bad[7, 0] = True
    assert torch.isnan(got[0][bad]).all() and torch.isfinite(got[0][~bad]).all() and not got[0, 9].any()
    assert (got[0, 11, 0] == 0).all()
    off = (got[0][~bad] - k[0][~bad]).abs() / k[0][~bad].abs().amax(-1, keepdim=True).clamp(min=1e-30)
    # half a step: of 127 parts, or 2^-4 of the number and half of the smallest, 2^-10 of 448
    assert off.max() <= (0.5 / 127 if store == "int8" else 2.0 ** -4) * 1.001
    # a query that sees a NaN row is NaN, one of the other head is not
    q = torch.randn(1, 1, 2, 64, device="cuda")
    out = P.pam_paged_attn(q, c.cache, c.table, ints([4]))
    assert torch.isnan(out[0, 0, 1]).all() and torch.isfinite(out[0, 0, 0]).all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_cache_write_strides(t):
    """New rows as parts of one projection, element by element and wide, sequences in any order."""
    import torch

    import paper_1907_00641_amd as P

    for off in (0, 1):
        a, b = Cache(44, 3, 30, 16, 2, 64, 64, t, "e4m3"), Cache(44, 3, 30, 16, 2, 64, 64, t, "e4m3")
        both = torch.randn(4, 3, 2 * 128 + 8, device="cuda").to(dt(t))
        k = both[:, :, off:off + 128].view(4, 3, 2, 64).transpose(0, 1)
        v = both[:, :, off + 128:off + 256].view(4, 3, 2, 64).transpose(0, 1)
        P.pam_cache_write(a.cache, k, v, a.table, a.k_len)
        P.pam_cache_write(b.cache, k.contiguous(), v.contiguous(), b.table, b.k_len)
        assert same((a.cache.k, a.cache.v, a.cache.k_scale, a.cache.v_scale),
                    (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale))


# ---------------------------------------------------------------------------
# attention over the cache
# ---------------------------------------------------------------------------

class Paged(Cache):
    def __init__(self, seed, B, n, total, page, H, hk, d, dv, t, store, maps=1, k_len=None, q_len=None, spread=1.0):
        super().__init__(seed, B, total, page, hk, d, dv, t, store, maps, k_len)
        rng = np.random.default_rng(seed + 1)
        shape = (B, n, H, 2, d) if maps == 2 else (B, n, H, d)
        self.q, self.qh = dev(spread * rng.standard_normal(shape), t)
        self.lam, self.lamh = dev(rng.uniform(0.2, 0.8, H), t) if maps == 2 else (None, None)
        self.q_len = q_len

    def run(self, **kw):
        import paper_1907_00641_amd as P

        return P.pam_paged_attn(self.q, self.cache, self.table, self.k_len, lam=self.lam,
                                q_len=None if self.q_len is None else ints(self.q_len), **kw)

    def compare(self, out):
        Paged.compare_with(self, self.q, self.qh, self.lamh, self.lam, self.q_len, out)

    @staticmethod
    def compare_with(c, q, qh, lamh, lam, q_len, out):
        n = int(np.clip(c.k_len_h, 0, c.table_h.shape[1] * c.page).max(initial=0))
        k, v, live = c.gathered(n)
        d, scale = c.d, c.d ** -0.5
        qh = qh.reshape(*qh.shape[:3], c.maps, d)
        want, mag = O.paged(qh, k, v, live, np.clip(c.k_len_h, 0, c.table_h.shape[1] * c.page), q_len, lamh, scale)
        S = scale * np.linalg.norm(qh, axis=-1).max(initial=0) * np.linalg.norm(k, axis=-1).max(initial=0)
        u, e = U[c.t], E * (2 * (c.maps * d + 6) * S + 20 + n)
        rounded = 2 if c.t == "f16" and c.store != c.t else 1
        # fp16: a probability under 2^-7 2^-14 of the largest has no relative precision left
        low = 2.0 ** -24 * np.abs(v).max(initial=0) * n if c.t == "f16" else 0.0
        check("out", out, want, u * np.abs(want) + (rounded * u + e) * mag + low * 2.0 ** -7 + TINY[c.t])


PAGED = [  # B, n, total, page, H, hk, d, dv, maps
    (1, 1, 1, 1, 1, 1, 16, 16, 1), (2, 1, 33, 16, 8, 2, 64, 64, 1), (1, 3, 100, 24, 4, 4, 40, 24, 1),
    (2, 1, 300, 5, 7, 1, 128, 128, 1), (1, 5, 70, 32, 14, 2, 64, 128, 2), (2, 2, 129, 8, 3, 3, 20, 40, 2),
    (1, 1, 65, 16, 2, 1, 7, 5, 1), (1, 2, 90, 64, 4, 2, 128, 256, 2), (1, 1, 40, 16, 2, 1, 256, 200, 1),
    (2, 40, 90, 16, 4, 2, 32, 64, 1), (3, 9, 50, 16, 16, 1, 64, 64, 2),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("shape", PAGED, ids=str)
def test_paged_attention_matches_oracle(shape, store, t):
    log(f"[paged] {shape} {store} {t}")
    B, n, total, page, H, hk, d, dv, maps = shape
    c = Paged(51, B, n, total, page, H, hk, d, dv, t, stored_as(t, store), maps,
              k_len=[total - 7 * b if total > 7 * b else 1 for b in range(B)])
    c.compare(c.run())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("maps", [1, 2])
def test_paged_attention_in_parts(store, t, maps):
    """A long axis, cut into parts that are joined, some of which see nothing; with bounds that cut it less."""
    log(f"[paged parts] {store} {t} maps={maps}")
    c = Paged(52, 3, 2, 5000, 16, 8, 2, 64, 64, t, stored_as(t, store), maps, k_len=[5000, 40, 1777])
    want = c.run()
    c.compare(want)
    for bound in (1, 600, 100000):
        c.compare(c.run(key_bound=bound))


@pytest.mark.parametrize("lens", [[4000, 1, 0, 17, 900, 2300], [1] * 5 + [6000], [1500] * 6, [300 + 61 * b for b in range(64)],
                                  [700 - 7 * b for b in range(70)], [0, 0, 0]], ids=["mixed", "one long", "equal", "64", "70", "none"])
@pytest.mark.parametrize("maps", [1, 2])
def test_paged_attention_shares(lens, maps):
    """The blocks are shared out by the sequences' lengths, which the host does not know; the bits do not depend on how
    much longer the table is, but for the split."""
    total = max(max(lens), 1) + 900
    c = Paged(59, len(lens), 1, total, 16, 4, 2, 32, 32, "bf16", "int8", maps, k_len=lens)
    want = c.run()
    c.compare(want)
    assert same(c.run(), want)
    c.compare(c.run(key_bound=max(max(lens), 1)))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("q_len,k_len", [([3, 0, 1], [20, 5, 9]), ([3, 3, 3], [2, 0, 3]), ([-1, 99, 2], [-4, 99999, 1])], ids=str)
@pytest.mark.parametrize("maps", [1, 2])
def test_paged_attention_lengths(q_len, k_len, t, maps):
    """Rows from q_len on and rows that see nothing are 0: new tokens at positions before the first, empty caches."""
    c = Paged(53, 3, 3, 40, 8, 4, 2, 32, 32, t, "int8", maps, k_len=k_len, q_len=q_len)
    out = c.run()
    c.compare(out)
    nq = np.clip(q_len, 0, 3)
    kl = np.clip(k_len, 0, 40)
    for b in range(3):
        for i in range(3):
            if i >= nq[b] or i + kl[b] - nq[b] < 0:
                assert not host(out)[b, i].any()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("d,maps", [(64, 1), (64, 2), (40, 1), (128, 2)])
def test_paged_attention_unused_places_may_hold_anything(store, t, d, maps):
    """NaN in pages that are no sequence's, behind the sequences' ends and in queries from q_len on: the same bits."""
    import torch

    c = Paged(54, 2, 3, 700, 16, 4, 2, d, d, t, stored_as(t, store), maps, k_len=[700, 301], q_len=[3, 2])
    want = c.run()
    free = torch.ones(c.pages, c.page, dtype=torch.bool, device="cuda")
    for b, n in enumerate(c.k_len_h):
        for p in range(n):
            free[c.table_h[b, p // c.page], p % c.page] = False
    free = free[:, None].expand(-1, c.hk, -1)
    for x in (c.cache.k, c.cache.v):
        if c.cache.k_scale is None:
            x[free] = float("nan")
        elif x.dtype is not torch.int8:
            x.view(torch.uint8)[free] = 0x7F  # NaN
    for x in (c.cache.k_scale, c.cache.v_scale):
        if x is not None:
            x[free] = float("nan")
    c.q[1, 2] = float("nan")
    assert same(c.run(), want)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_paged_attention_is_the_contiguous_one(t):
    """One map: pam_attn_fwd over the same keys; two: pam_diff_attn_fwd; within what rounding probabilities allows."""
    import paper_1907_00641_amd as P

    for maps in (1, 2):
        c = Paged(55, 2, 4, 333, 16, 6, 2, 64, 128, t, t, maps, k_len=[333, 70])
        got = host(c.run())
        k, v = P.pam_cache_read(c.cache, c.table, c.k_len, 333)
        if maps == 2:
            want = host(P.pam_diff_attn_fwd(c.q, k, v, c.lam, causal=True, k_len=c.k_len))
        else:
            want = np.stack([host(P.pam_attn_fwd(c.q[b], k[b, :n], v[b, :n], causal=True)) for b, n in enumerate(c.k_len_h)])
        assert np.abs(got - want).max() <= 4 * U[t] * np.abs(c.vn).max() + 1e-5


@pytest.mark.parametrize("store", STORES)
def test_paged_attention_large_scores_and_scales(store):
    """Scores of some hundreds; in fp16 values whose scales are of 1e-4 and 100."""
    c = Paged(56, 1, 2, 200, 16, 4, 2, 64, 64, "f16", stored_as("f16", store), spread=30.0)
    c.compare(c.run())
    rng = np.random.default_rng(57)
    size = np.exp2(rng.uniform(-13, 8, (c.pages, 2, 16, 1)))
    c.fill(rng.standard_normal((c.pages, 2, 16, 64)), np.float16(rng.standard_normal((c.pages, 2, 16, 64)) * size))
    c.compare(c.run())


@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_paged_attention_value_scales(store, order):
    """Values from 2^-30 to 2^30 over the keys of a sequence: scales go into the product relative to the largest so far."""
    c = Paged(60, 2, 2, 400, 16, 4, 2, 64, 64, "bf16", store, k_len=[400, 333])
    rng = np.random.default_rng(61)
    size = np.ones((c.pages, 2, 16, 1))
    for b in range(2):
        for p in range(400):
            e = {"rising": p / 400 * 60 - 30, "falling": 30 - p / 400 * 60, "mixed": rng.uniform(-30, 30)}[order]
            size[c.table_h[b, p // 16], :, p % 16] = 2.0 ** e
    c.fill(rng.standard_normal((c.pages, 2, 16, 64)), rng.standard_normal((c.pages, 2, 16, 64)) * size)
    out = c.run()
    k, v, live = c.gathered(400)
    want, mag = O.paged(c.qh.reshape(2, 2, 4, 1, 64), k, v, live, c.k_len_h, None, None, 0.125)
    S = 0.125 * np.linalg.norm(c.qh, axis=-1).max() * np.linalg.norm(k, axis=-1).max()
    # a product of a probability and a scale: 11 bits, or 2^-31 of the largest scale, whose numbers reach
    # the largest value; a sum of probabilities is at least 1
    tol = U["bf16"] * np.abs(want) + (U["f16"] + E * (2 * 70 * S + 420)) * mag + 400 * 2.0 ** -31 * np.abs(v).max()
    check("out", out, want, tol + TINY["bf16"])


def test_paged_attention_strides_streams_graph():
    """Queries as a part of a projection; another stream; captured, the lengths growing between replays."""
    import torch

    import paper_1907_00641_amd as P

    c = Paged(58, 2, 1, 900, 16, 8, 2, 64, 64, "bf16", "e4m3", k_len=[850, 400])
    want = c.run()
    for off in (0, 3):
        wide = torch.full((2, 1, 8 * 64 + 16), float("nan"), dtype=torch.bfloat16, device="cuda")
        q = wide[:, :, off:off + 512].view(2, 1, 8, 64)
        q.copy_(c.q)
        assert same(P.pam_paged_attn(q, c.cache, c.table, c.k_len), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(stream=side)
    side.synchronize()
    assert same(got, want) and same(c.run(), want)
    new = torch.randn(2, 1, 2, 64, device="cuda").to(torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.pam_cache_write(c.cache, new, new, c.table, c.k_len)
        out = P.pam_paged_attn(c.q, c.cache, c.table, c.k_len)
    for step in range(4):
        c.k_len += 1
        c.q.add_(0.1)
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, P.pam_paged_attn(c.q, c.cache, c.table, c.k_len)), step


def test_paged_far_offsets():
    """Rows whose offsets pass 2^32 bytes in the pool."""
    import torch

    import paper_1907_00641_amd as P

    page, hk, d = 16, 1, 128
    pages = (1 << 32) // (page * d) + 50
    k = torch.empty(pages, hk, page, d, dtype=torch.int8, device="cuda")
    v, ks, vs = torch.empty_like(k), torch.empty(pages, hk, page, device="cuda"), torch.empty(pages, hk, page, device="cuda")
    far = P.PagedCache(k, v, ks, vs)
    near = P.PagedCache.empty(8, page, hk, d, dtype=torch.int8)
    rows = torch.randn(1, 100, hk, d, device="cuda").to(torch.bfloat16)
    q = torch.randn(1, 2, 4, d, device="cuda").to(torch.bfloat16)
    res = []
    for cache, first in ((far, pages - 7), (near, 0)):
        table = (torch.arange(7, dtype=torch.int32, device="cuda") + first)[None]
        P.pam_cache_write(cache, rows, rows * 0.5, table, ints([100]))
        res.append((*P.pam_cache_read(cache, table, ints([100]), 100, dtype=torch.bfloat16),
                    P.pam_paged_attn(q, cache, table, ints([100]))))
    assert same(*res)
    del k, v, ks, vs, far
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("store", ["bf16", "e4m3", "int8"])
def test_prompt_and_decoding_together(store):
    """Queries and keys normed and turned, prompts of different lengths attended to packed and written to the cache,
    then token by token; against the packed attention over what the cache holds, sequence by sequence."""
    import torch

    import paper_1907_00641_amd as P

    gen = torch.Generator(device="cuda")
    gen.manual_seed(61)
    H, hk, d, page, prompts, steps = 8, 2, 64, 16, [70, 1, 133], 20
    total = [n + steps for n in prompts]

    def normal(*s):
        return torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)

    data = [(normal(n, H, d), normal(n, hk, d), normal(n, hk, d)) for n in total]
    freq, mag = P.pam_rotary_frequencies(d)
    table = P.pam_rotary_table(freq.cuda(), entries=max(total), magnitude=mag)
    w = torch.rand(d, generator=gen, device="cuda") + 0.5
    cache = P.PagedCache.empty(40, page, hk, d, dtype=store_type(store))
    pages = torch.randperm(40, generator=torch.Generator().manual_seed(5))[:30].reshape(3, 10).to(torch.int32).cuda()

    def turned(q, k, pos):
        q, k = P.pam_head_norm_rotary_fwd(q[None], k[None], table, w_q=w, w_k=w, pos=ints(pos)[None])
        return q[0], k[0]

    starts = ints(np.concatenate([[0], np.cumsum(prompts)]))
    q, k = turned(*(torch.cat([x[i][:n] for x, n in zip(data, prompts)]) for i in (0, 1)),
                  np.concatenate([np.arange(n) for n in prompts]))
    v = torch.cat([x[2][:n] for x, n in zip(data, prompts)])
    out = P.pam_attn_fwd(q, k, v, q_start=starts, k_start=starts, causal=True)
    P.pam_cache_write(cache, k, v, pages, ints(prompts), starts=starts)
    got = [[out[a:b]] for a, b in zip(np.cumsum([0] + prompts[:-1]), np.cumsum(prompts))]
    for s in range(steps):
        at = [n + s for n in prompts]
        q, k = turned(*(torch.stack([x[i][n] for x, n in zip(data, at)]) for i in (0, 1)), at)
        v = torch.stack([x[2][n] for x, n in zip(data, at)])
        n = ints([n + 1 for n in at])
        P.pam_cache_write(cache, k[:, None], v[:, None], pages, n)
        o = P.pam_paged_attn(q[:, None], cache, pages, n)
        for b in range(3):
            got[b].append(o[b])
    rk, rv = P.pam_cache_read(cache, pages, ints(total), max(total), dtype=torch.bfloat16)
    for b, n in enumerate(total):
        q, k = turned(data[b][0], data[b][1], np.arange(n))
        if store == "bf16":
            assert same(rk[b, :n], k) and same(rv[b, :n], data[b][2])
        whole = P.pam_attn_fwd(q, rk[b, :n], rv[b, :n], causal=True)
        tail = torch.cat(got[b])[prompts[b]:]
        # the values read back are rounded to bf16 here and exact there: u of the largest value, and u for the
        # probabilities and the result on either side; keys that are rounded move scores of up to |q| |k| / 8 by u
        score = float(q.float().norm(dim=-1).max() * rk[b].float().norm(dim=-1).max()) / 8
        off = (tail.float() - whole[prompts[b]:].float()).abs().max().item()
        bound = U["bf16"] * (5 + 2 * (0 if store == "bf16" else score)) * rv[b].abs().max().item()
        log(f"  {store}, sequence {b}: off by {off:.4f}, bound {bound:.4f}")
        assert off <= bound
