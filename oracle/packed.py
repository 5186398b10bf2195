"""Oracle of attention over packed sequences and from a paged cache
(include/pam_packed.h), in numpy and 64 bits: the plain definitions, gradients
by formula, and, for every result, the sum of the absolute values of the terms
it is made of, from which the tests derive how far a computation in fewer bits
may be off.
"""
import numpy as np

TOP = {"e4m3": 448.0, "int8": 127.0}


# ---------------------------------------------------------------------------
# attention with one softmax map
# ---------------------------------------------------------------------------

def _softmax(s, see):
    """Rows of probabilities, 0 where nothing is seen, and the logarithm of the sums."""
    s = np.where(see, s, -np.inf)
    top = s.max(axis=-1, keepdims=True, initial=-np.inf)
    top = np.where(np.isfinite(top), top, 0.0)
    e = np.where(see, np.exp(s - top), 0.0)
    total = e.sum(axis=-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.log(total[..., 0]) + top[..., 0]
    return np.divide(e, total, out=np.zeros_like(e), where=total > 0), lse


def sequence(q, k, v, scale, see, g=None):
    """One head of one sequence: q n x d, k m x d, v m x dv, see n x m.  Returns (results, magnitudes) by name: out,
    lse, and from the upstream gradient g dq, dk, dv.  A gradient's magnitudes: of |ds|, of p |D| and of p |dp|."""
    p, lse = _softmax(scale * (q @ k.T), see)
    r, a = {"out": p @ v, "lse": lse}, {"out": p @ np.abs(v)}
    if g is None:
        return r, a
    dp, dp_abs = g @ v.T, np.abs(g) @ np.abs(v).T
    D = (g * r["out"]).sum(axis=1, keepdims=True)
    D_abs = (np.abs(g) * a["out"]).sum(axis=1, keepdims=True)
    ds = scale * p * (dp - D)
    parts = (np.abs(ds), scale * p * D_abs, scale * p * dp_abs)
    r.update(dq=ds @ k, dk=ds.T @ q, dv=p.T @ g)
    a.update(dq=[x @ np.abs(k) for x in parts], dk=[x.T @ np.abs(q) for x in parts], dv=p.T @ np.abs(g))
    return r, a


def causal(n, m):
    """Which of m keys each of n queries sees: the last query sees all."""
    return np.arange(m)[None] <= np.arange(n)[:, None] + m - n


def packed(q, k, v, scale, q_ends, k_ends, is_causal, g=None):
    """Packed sequences: q T x H x d, k S x Hk x d, v S x Hk x dv, sequence b the rows ends[b] .. ends[b + 1] - 1.
    Returns (results, magnitudes) of the arrays' shapes; 0 in rows of no sequence."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    (T, H, d), (S, hk, dv) = q.shape, v.shape
    r = {"out": np.zeros((T, H, dv)), "lse": np.full((H, T), -np.inf), "dq": np.zeros_like(q), "dk": np.zeros_like(k),
         "dv": np.zeros_like(v)}
    a = {"out": np.zeros((T, H, dv)), "dv": np.zeros_like(v), "dq": [np.zeros_like(q) for _ in range(3)],
         "dk": [np.zeros_like(k) for _ in range(3)]}
    for b in range(len(q_ends) - 1):
        x, y = slice(q_ends[b], q_ends[b + 1]), slice(k_ends[b], k_ends[b + 1])
        n, m = q_ends[b + 1] - q_ends[b], k_ends[b + 1] - k_ends[b]
        see = causal(n, m) if is_causal else np.ones((n, m), dtype=bool)
        for h in range(H):
            c = h // (H // hk)
            s, t = sequence(q[x, h], k[y, c], v[y, c], scale, see, None if g is None else np.asarray(g, np.float64)[x, h])
            r["out"][x, h], r["lse"][h, x], a["out"][x, h] = s["out"], s["lse"], t["out"]
            if g is None:
                continue
            r["dq"][x, h] = s["dq"]
            r["dk"][y, c] += s["dk"]
            r["dv"][y, c] += s["dv"]
            a["dv"][y, c] += t["dv"]
            for i in range(3):
                a["dq"][i][x, h] = t["dq"][i]
                a["dk"][i][y, c] += t["dk"][i]
    return r, a


# ---------------------------------------------------------------------------
# norms of heads, rotary positions
# ---------------------------------------------------------------------------

def _turn(x, cos, sin, interleaved, sign):
    n = cos.shape[-1]
    c, s = cos[:, :, None], sign * sin[:, :, None]
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y = np.array(x)
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., first] * s + x[..., second] * c
    return y


def _turn_abs(x, cos, sin, interleaved):
    return np.abs(_turn(np.abs(x), np.abs(cos), -np.abs(sin), interleaved, 1.0)) + \
        np.abs(_turn(np.abs(x), np.abs(cos), np.abs(sin), interleaved, 1.0))


def head_norm(x, w, cos, sin, layer, eps, interleaved, g=None):
    """x: B x L x H x d; w: d or H x d; cos, sin: B x L x pairs, of each token.  Returns (results, magnitudes) by name:
    y and, from the upstream gradient g, dx and dw."""
    x = np.asarray(x, dtype=np.float64)
    z = x - x.mean(-1, keepdims=True) if layer else x
    r = 1.0 / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
    n = z * r
    # what a mean that is taken in fewer bits leaves of the row
    n_abs = (np.abs(x) + (np.abs(x).mean(-1, keepdims=True) if layer else 0.0)) * r
    res = {"y": _turn(n * w, cos, sin, interleaved, 1.0)}
    mag = {"y": _turn_abs(n_abs * w, cos, sin, interleaved)}
    if g is None:
        return res, mag
    dy = _turn(np.asarray(g, dtype=np.float64), cos, sin, interleaved, -1.0)
    dy_abs = _turn_abs(g, cos, sin, interleaved)
    dn, dn_abs = dy * w, dy_abs * np.abs(w)
    dx = dn - n * (dn * n).mean(-1, keepdims=True)
    dx_abs = dn_abs + n_abs * (dn_abs * n_abs).mean(-1, keepdims=True)
    if layer:
        dx = dx - dn.mean(-1, keepdims=True)
        dx_abs = dx_abs + dn_abs.mean(-1, keepdims=True)
    over = (0, 1) if np.ndim(w) == 2 else (0, 1, 2)
    res.update(dx=dx * r, dw=(dy * n).sum(over))
    mag.update(dx=dx_abs * r, dw=(dy_abs * n_abs).sum(over))
    return res, mag


# ---------------------------------------------------------------------------
# the paged cache
# ---------------------------------------------------------------------------

def stored(x, store):
    """Numbers and scales of rows (last axis) that are stored in 8 bits; quotients rounded to fp32 (a correctly
    rounded 64-bit quotient of fp32 numbers, rounded to fp32, is the correctly rounded fp32 one)."""
    x = np.asarray(x, dtype=np.float64)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    scale = np.maximum((np.abs(x).max(-1) / TOP[store]).astype(np.float32), np.float32(2.0 ** -126))
    y = (x / scale[..., None].astype(np.float64)).astype(np.float32).astype(np.float64)
    y = np.clip(y, -TOP[store], TOP[store])
    if store == "e4m3":
        step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
        y = np.rint(y / step) * step
    else:
        y = np.rint(y)
    return y, np.where(bad, np.float32(np.nan), scale)


def places(table, pages, page, length):
    """Page and place of positions 0 .. length - 1 of every sequence; page -1 where there is none."""
    p = np.arange(length)
    at = np.asarray(table)[:, p // page]
    return np.where((at >= 0) & (at < pages), at, -1), p % page


def gathered(values, table, page, k_len, length):
    """values: pages x Hk x page x ...; the first ``length`` positions of every sequence, 0 where there is no token,
    and which there are."""
    at, off = places(table, values.shape[0], page, length)
    live = (at >= 0) & (np.arange(length)[None] < np.clip(k_len, 0, table.shape[1] * page)[:, None])
    got = values[np.where(live, at, 0), :, off[None]]
    return np.where(live.reshape(*live.shape, *([1] * (got.ndim - 2))), got, 0.0), live


def paged(q, k, v, live, k_len, q_len, lam, scale):
    """q: B x L x H x maps x d; k: B x n x Hk x maps x d and v: B x n x Hk x dv as gathered; live B x n.  Returns the
    output and its magnitude."""
    q = np.asarray(q, dtype=np.float64)
    B, L, H, maps, d = q.shape
    n, hk, dv = v.shape[1:]
    out, mag = np.zeros((B, L, H, dv)), np.zeros((B, L, H, dv))
    for b in range(B):
        nq = L if q_len is None else min(max(int(q_len[b]), 0), L)
        last = np.arange(L)[:, None] + int(k_len[b]) - nq
        see = (np.arange(n)[None] <= last) & live[b][None] & (np.arange(L)[:, None] < nq)
        for h in range(H):
            c = h // (H // hk)
            for m in range(maps):
                r, a = sequence(q[b, :, h, m], k[b, :, c, m], v[b, :, c], scale, see)
                f = 1.0 if m == 0 else -float(lam[h])
                out[b, :, h] += f * r["out"]
                mag[b, :, h] += abs(f) * a["out"]
    return out, mag
