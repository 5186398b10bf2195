"""Edges of attention over packed sequences and of the paged cache that test_packed_gpu.py leaves out: values of a few
small sizes behind pages that are not there.  Bounds as there."""
import numpy as np
import pytest

from helpers import log
from oracle import packed as O
from test_attn_gpu import TINY, U, _cuda, check  # noqa: F401
from test_packed_gpu import E, Paged

pytestmark = pytest.mark.gpu


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
