"""Edges of attention over packed sequences and of the paged cache that test_packed_gpu.py leaves out: starts that fall,
lengths past the table, small values beside pages that are not there, and results that are off by their own rounding
alone.  Bounds as there."""
import numpy as np
import pytest

from helpers import log
from oracle import packed as O
from test_attn_gpu import TINY, U, _cuda, check, dev, dt, host  # noqa: F401
from test_packed_gpu import Cache, E, Packed, Paged, ints, numbers, same, stored_as

pytestmark = pytest.mark.gpu


def own_rounding(name, got, want, t, rest):
    """Whether ``got`` is off by no more than by being rounded to its type when it is stored, of the norm.

    ``want`` rounded to the type is off by e, and the kernel's values, which differ from ``want`` by less than a step,
    are when they are rounded, but for chance: 2 / sqrt(N) of it over N values.  ``rest`` is how far they are off before that,
    which adds at random, in squares.  An operand that is rounded to the type alone would make it 1.41 e and more: its
    terms are off by as much as the result's values are by their rounding, and their squares add up to more than its own."""
    import torch

    e = np.linalg.norm(torch.from_numpy(want).to(dt(t)).double().numpy() - want)
    off, n = np.linalg.norm(host(got) - want), want.size
    log(f"  {name}: off by {off / e:.3f} times its own rounding, {rest / e:.3f} before it")
    assert n >= 3000 and rest < 0.6 * e and off <= (1 + 2 / np.sqrt(n)) * np.hypot(e, rest), (name, off / e)


# ---------------------------------------------------------------------------
# attention over packed sequences
# ---------------------------------------------------------------------------

def sequences(c):
    """Queries, keys and who sees whom, of each sequence."""
    for b in range(len(c.q_ends) - 1):
        x, y = slice(c.q_ends[b], c.q_ends[b + 1]), slice(c.k_ends[b], c.k_ends[b + 1])
        n, m = x.stop - x.start, y.stop - y.start
        yield x, y, O.causal(n, m) if c.causal else np.ones((n, m), dtype=bool)


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,d", [([300, 137], 64), ([300, 137], 40), ([500], 16), ([140] * 40, 32)], ids=str)
def test_attention_grad_q_is_rounded_once(lens, d, causal, t):
    """Heads of up to 64: score gradients enter their product with what their rounding leaves, u^2 of them."""
    log(f"[packed dq] {lens[:3]} {d} {t} causal={causal}")
    c = Packed(68, lens, 20, 4, 2, d, d, t, causal)
    (_, dq, _, _), _ = c.run()
    r, _ = O.packed(c.qh, c.kh, c.vh, c.scale, c.q_ends, c.k_ends, causal, c.gh)
    S = c.scale * np.linalg.norm(c.qh, axis=-1).max() * np.linalg.norm(c.kh, axis=-1).max()
    # 32-bit sums at random: of a score of up to S and of dp over d products, of a row and a column over n keys, an
    # exponential; the squares of a value's terms, of zero mean, add up to 1.0 to 1.3 times its own (as numpy has them)
    n = max(lens) + 20
    rest = 1.2 * (E * (np.sqrt(d + 6) * S + np.sqrt(d + 8) + np.sqrt(n) + 8) + U[t] ** 2) * np.linalg.norm(r["dq"])
    # D is of out as the forward pass saves it, whose probabilities are rounded to the type: off by at most u each,
    # u^2 / 3 in squares, D_i by the root of sum u^2 / 3 (p_ij dp_ij)^2, and dq_i by that times scale sum p_ij k_j
    square = 0.0
    for x, y, see in sequences(c):
        for h in range(4):
            p, _ = O._softmax(c.scale * c.qh[x, h] @ c.kh[y, h // 2].T, see)
            dp = c.gh[x, h] @ c.vh[y, h // 2].T
            square += (((p * dp) ** 2).sum(1) * ((p @ c.kh[y, h // 2]) ** 2).sum(1)).sum()
    rest = np.hypot(rest, c.scale * U[t] * np.sqrt(square / 3))
    own_rounding("dq", dq, r["dq"], t, rest)


def compare_short(c, results):
    """As Packed.compare, and with a term that only counts where a sequence has few keys: D is of out as the forward pass
    saves it, from probabilities that are rounded to the type, each by u: it is off by d_i = u sum_j p_ij |dp_ij| at the
    most, dq_i by d_i scale |sum_j p_ij k_j|, and dk_j by scale sum_i d_i p_ij |q_i|."""
    r, a = O.packed(c.qh, c.kh, c.vh, c.scale, c.q_ends, c.k_ends, c.causal, c.gh)
    u, tiny, (_, H, d), hk = U[c.t], TINY[c.t], c.qh.shape, c.kh.shape[1]
    by_d = {"dq": np.zeros_like(c.qh), "dk": np.zeros_like(c.kh)}
    for x, y, see in sequences(c):
        for h in range(H):
            k = h // (H // hk)
            p, _ = O._softmax(c.scale * c.qh[x, h] @ c.kh[y, k].T, see)
            off = u * (p * np.abs(c.gh[x, h] @ c.vh[y, k].T)).sum(1, keepdims=True)
            by_d["dq"][x, h] = off * c.scale * np.abs(p @ c.kh[y, k])
            by_d["dk"][y, k] += c.scale * (p * off).T @ np.abs(c.qh[x, h])
    lk, lq = int(np.diff(c.k_ends).max()), int(np.diff(c.q_ends).max()) * (H // hk)
    S = c.scale * np.linalg.norm(c.qh, axis=-1).max() * np.linalg.norm(c.kh, axis=-1).max()
    e, ep = E * (2 * (d + 6) * S + 16 + lk), E * (c.vh.shape[-1] + 8)
    check("out", results[0], r["out"], u * np.abs(r["out"]) + (u + e) * a["out"] + tiny)
    for name, got, n in (("dq", results[1], lk), ("dk", results[2], lq)):
        A0, AD, AP = a[name]
        check(name, got, r[name], u * np.abs(r[name]) + (u + e + n * E) * A0 + (2 * e + ep) * (AD + AP) + by_d[name] + tiny)
    check("dv", results[3], r["dv"], u * np.abs(r["dv"]) + (u + e + lq * E) * a["dv"] + tiny)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("count", [256, 257, 1000, 4097])
def test_attention_very_many_sequences(count, causal, t):
    """Places found by looking through the sequences, and among sums of their tiles; of no row, of one, of a tile and of
    several; replayed from a graph with other lengths in the same starts."""
    import torch

    import paper_1907_00641_amd as P

    log(f"[packed] {count} sequences {t} causal={causal}")
    rng = np.random.default_rng(count)
    lens = [int(x) for x in rng.choice([0, 1, 5, 17, 40], count)]
    for i, n in ((0, 129), (3, 256), (count // 2, 300), (count - 1, 130)):
        lens[i] = n
    c = Packed(70, lens, 1, 2, 1, 24, 24, t, causal, before=3, behind=5)
    res, _ = c.run()
    compare_short(c, res)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, s = P.pam_attn_fwd(c.q, c.k, c.v, save=True, **c.how)
        grads = P.pam_attn_bwd(c.q, c.k, c.v, s, c.g, **c.how)
    for ends in (c.q_ends, [n // 2 for n in c.q_ends], c.q_ends):
        c.how["q_start"].copy_(ints(ends))
        c.how["k_start"].copy_(ints(ends))
        for _ in range(2):
            graph.replay()
            torch.cuda.synchronize()
            assert same((out, *grads), c.run()[0])


class Guarded:
    """Arrays with 4 KB before and behind each that nothing may change."""

    def __init__(self):
        self.all = []

    def array(self, shape, dtype):
        import torch

        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        raw = torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        self.all.append((raw, n))
        return raw[4096:4096 + n].view(dtype).view(*shape)

    def untouched(self):
        return all((raw[:4096] == 0xA5).all() and (raw[4096 + n:] == 0xA5).all() for raw, n in self.all)


def guarded_attention(c, q_start, k_start):
    """Forward and backward through the C ABI on guarded arrays: (out, grads), and whether the guards are whole."""
    import ctypes

    import torch

    from paper_1907_00641_amd import binding as B

    desc, ptrs, _ = B._attn_desc(c.q, c.k, c.v, q_start, k_start, c.scale, c.causal)
    L, d, g = B.lib(), ctypes.byref(desc), Guarded()
    (T, H, _), f32 = c.q.shape, torch.float32
    out, so, lse = g.array(c.g.shape, c.q.dtype), g.array(c.g.shape, f32), g.array((H, T), f32)
    grads = [g.array(x.shape, x.dtype) for x in (c.q, c.k, c.v)]
    ws = [g.array((max(f(d), 16),), torch.uint8) for f in (L.pam_attn_fwd_workspace, L.pam_attn_bwd_workspace)]
    s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert L.pam_attn_fwd(d, *ptrs, out.data_ptr(), so.data_ptr(), lse.data_ptr(), ws[0].data_ptr(), s) == B.PAM_OK
    assert L.pam_attn_bwd(d, *ptrs, so.data_ptr(), lse.data_ptr(), c.g.data_ptr(), (ctypes.c_int64 * 2)(*c.g.stride()[:2]),
                          *(x.data_ptr() for x in grads), ws[1].data_ptr(), s) == B.PAM_OK
    torch.cuda.synchronize()
    return (out, *grads), g.untouched()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 72])
def test_attention_starts_that_fall(d, causal, t):
    """Sequences that would end before they start are empty, up to 64 of them and more: where no row is a sequence's, all
    results are 0; where sequences lie over each other, nothing beside the arrays is written, forward or backward."""
    rng = np.random.default_rng(66)
    c = Packed(67, [300, 137], 0, 4, 2, d, d, t, causal)
    for count in (2, 64, 65, 200, 300, 9000):
        falls = np.linspace(400, 0, count + 1).astype(int)
        log(f"[falling starts] {count} sequences, all empty, {d} {t} causal={causal}")
        res, whole = guarded_attention(c, ints(falls), ints(falls))
        assert whole and not any(x.any() for x in res)
        over = rng.integers(0, 438, count + 1)
        over[::7] = rng.choice([-2 ** 31, 2 ** 31 - 1, 437, 0], len(over[::7]))
        log(f"[falling starts] {count} sequences over each other")
        assert guarded_attention(c, ints(over), ints(over[::-1].copy()))[1]
        assert guarded_attention(c, ints(over), ints(np.linspace(0, 437, count + 1).astype(int)))[1]
    ends = ints([0, 300, 437])
    res, whole = guarded_attention(c, ends, ends)
    assert whole
    c.compare(res)


# ---------------------------------------------------------------------------
# the paged cache
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 20])
@pytest.mark.parametrize("how", ["padded", "ragged", "packed"])
def test_cache_writes_past_the_table(how, d, store, t):
    """New tokens whose positions the table does not reach are not written, and write no other's place: lengths one past
    the table, past it by more than the new tokens, the largest number; and all in it.  Every number and scale of the
    pool, as the oracle stores them."""
    import torch

    import paper_1907_00641_amd as P

    log(f"[cache past the table] {how} {d} {store} {t}")
    store, capacity = stored_as(t, store), 40
    k_len = np.array([capacity + 1, capacity + 9, 2 ** 31 - 1, capacity, capacity + 2])
    new_len = np.array([3, 3, 3, 3, 3] if how == "padded" else [2, 3, 1, 3, 0])
    c = Cache(64, 5, capacity, 8, 2, d, d, t, store, k_len=k_len)
    rng = np.random.default_rng(65)
    k, kh = dev(rng.standard_normal((5, 3, 2, d)), t)
    v, vh = dev(rng.standard_normal((5, 3, 2, d)), t)
    pools = ((kh, c.cache.k, c.cache.k_scale), (vh, c.cache.v, c.cache.v_scale))
    want = [(numbers(pool), None if scale is None else host(scale)) for _, pool, scale in pools]
    for b, n in enumerate(new_len):
        for i in range(n):
            p = int(k_len[b]) - n + i
            if p >= capacity:
                continue
            at = (c.table_h[b, p // 8], slice(None), p % 8)
            for (x, _, _), (num, sc) in zip(pools, want):
                if sc is None:
                    num[at] = x[b, i]
                else:
                    num[at], sc[at] = O.stored(x[b, i], store)
    if how == "packed":
        rows = [torch.cat([x[b, :n] for b, n in enumerate(new_len)]) for x in (k, v)]
        P.pam_cache_write(c.cache, *rows, c.table, c.k_len, starts=ints(np.concatenate([[0], np.cumsum(new_len)])))
    else:
        P.pam_cache_write(c.cache, k, v, c.table, c.k_len, new_len=None if how == "padded" else ints(new_len))
    for (_, pool, scale), (num, sc) in zip(pools, want):
        assert np.array_equal(numbers(pool), num)
        if sc is not None:
            assert np.array_equal(host(scale), sc)


# ---------------------------------------------------------------------------
# attention over the cache
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("t,size", [("bf16", 2.0 ** -20), ("bf16", 2.0 ** -30), ("f16", 2.0 ** -12)], ids=str)
@pytest.mark.parametrize("store", ["e4m3", "int8"])
@pytest.mark.parametrize("from_,to", [(0, 64), (32, 96)], ids=["first", "middle"])
@pytest.mark.parametrize("what", ["no page", "zeros"])
def test_paged_attention_small_values_beside_a_hole(what, from_, to, store, t, size):
    """Whole tiles of keys without a page, as a window that slides leaves them, or whose values' scales are 0, as
    PagedCache.empty has them, before and between keys with small values: those keep their precision."""
    log(f"[paged hole] {what} {from_}..{to} {store} {t} {size}")
    c = Paged(62, 2, 2, 400, 16, 4, 2, 64, 64, t, store, k_len=[400, 333])
    rng = np.random.default_rng(63)
    lead = (c.pages, 2, 16, 64)
    v = size * rng.standard_normal(lead)
    hole = slice(from_ // 16, to // 16)
    if what == "zeros":
        v[c.table_h[:, hole]] = 0.0
    c.fill(rng.standard_normal(lead), v)
    if what == "zeros":
        c.cache.v_scale[c.table[:, hole].long()] = 0.0
    else:
        c.table[:, hole] = -1
        c.table_h[:, hole] = -1
    out = c.run()
    k, v, live = c.gathered(400)
    want, mag = O.paged(c.qh.reshape(2, 2, 4, 1, 64), k, v, live, c.k_len_h, None, None, 0.125)
    S = 0.125 * np.linalg.norm(c.qh, axis=-1).max() * np.linalg.norm(k, axis=-1).max()
    # a product of a probability and a scale: 11 bits, or 2^-31 of the largest scale that is seen, whose numbers
    # reach the largest value; a sum of probabilities is at least 1
    tol = U[t] * np.abs(want) + (U["f16"] + E * (2 * 70 * S + 420)) * mag + 400 * 2.0 ** -31 * np.abs(v).max()
    check("out", out, want, tol + TINY[t])


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("store", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("maps,d,total", [(1, 64, 400), (2, 64, 400), (1, 128, 90), (1, 40, 3000)], ids=str)
def test_paged_attention_is_rounded_once(maps, d, total, store, t):
    """Pages of 16 bits, and of 8 with fp16: probabilities enter their product with what their rounding leaves; pages of
    8 bits with bf16: in fp16, 2^-11 of each term."""
    log(f"[paged] {maps} {d} {total} {store} {t}")
    c = Paged(69, 3, 2, total, 16, 16, 2, d, d * maps, t, stored_as(t, store), maps, k_len=[total, total // 2, total - 1])
    out = c.run()
    k, v, live = c.gathered(total)
    want, _ = O.paged(c.qh.reshape(3, 2, 16, maps, d), k, v, live, c.k_len_h, None, c.lamh, d ** -0.5)
    S = d ** -0.5 * np.linalg.norm(c.qh, axis=-1).max() * np.linalg.norm(k, axis=-1).max()
    rounded = U["f16"] if store != "same" and t == "bf16" else U[t] ** 2
    # as above; values are of zero mean
    rest = 1.2 * (E * (np.sqrt(maps * d + 6) * S + np.sqrt(total) + 8) + rounded) * np.linalg.norm(want)
    own_rounding("out", out, want, t, rest)
