"""Edges of attention over packed sequences and of the paged cache that test_packed_gpu.py leaves out: lengths past
the table, small values beside pages that are not there.  Bounds as there."""
import numpy as np
import pytest

from helpers import log
from oracle import packed as O
from test_attn_gpu import TINY, U, _cuda, check, dev, host  # noqa: F401
from test_packed_gpu import Cache, E, Paged, ints, numbers, stored_as

pytestmark = pytest.mark.gpu


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
