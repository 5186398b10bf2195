"""Oracle of the operators around an attention layer (include/pam_attn.h), in
numpy and 64 bits: the plain definitions, their gradients by formula, and, for
every result, the sum of the absolute values of the terms it is made of, from
which the tests derive how far a computation in fewer bits may be off.
"""
import numpy as np


# ---------------------------------------------------------------------------
# differential attention
# ---------------------------------------------------------------------------

def visible(B, lq, lk, causal, q_len=None, k_len=None, key_mask=None):
    """Which key each query sees: B x lq x lk."""
    see = np.zeros((B, lq, lk), dtype=bool)
    for b in range(B):
        nq = lq if q_len is None else min(max(int(q_len[b]), 0), lq)
        nk = lk if k_len is None else min(max(int(k_len[b]), 0), lk)
        for i in range(nq):
            last = min(nk, i + nk - nq + 1) if causal else nk
            if last > 0:
                see[b, i, :last] = True
        if key_mask is not None:
            see[b] &= np.asarray(key_mask[b], dtype=bool)[None, :]
    return see


def _softmax(s, see):
    """Rows of probabilities, 0 where nothing is seen, and the logarithm of the sums."""
    s = np.where(see, s, -np.inf)
    top = s.max(axis=-1, keepdims=True, initial=-np.inf)
    e = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0.0)), 0.0)
    total = e.sum(axis=-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = np.log(total[..., 0]) + np.where(np.isfinite(top), top, 0.0)[..., 0]
    return np.divide(e, total, out=np.zeros_like(e), where=total > 0), lse


def attention(q, k, v, lam, scale, see, grad_out=None):
    """Differential attention and, with ``grad_out``, its gradients.

    q: B x lq x H x 2 x d, k: B x lk x Hk x 2 x d, v: B x lk x Hk x dv, lam: H.
    Returns (results, magnitudes), dicts by name: out, o (2 x B x lq x H x dv),
    lse (2 x B x H x lq) and dq, dk, dv, dlam.  A magnitude is a list of terms:
    ``out`` [P |v|]; gradients [|ds| sums, D sums, dp sums] (see the tests)."""
    q, k, v, lam = (np.asarray(x, dtype=np.float64) for x in (q, k, v, lam))
    B, lq, H, _, d = q.shape
    lk, hk, dv = k.shape[1], k.shape[2], v.shape[3]
    G = H // hk
    # what no query of a sequence sees is no part of anything, whatever it holds
    used = see.any(axis=1)
    k = np.where(used[:, :, None, None, None], k, 0.0)
    v = np.where(used[:, :, None, None], v, 0.0)
    rows = see.any(axis=2)
    q = np.where(rows[:, :, None, None, None], q, 0.0)
    r = {"out": np.zeros((B, lq, H, dv)), "o": np.zeros((2, B, lq, H, dv)), "lse": np.zeros((2, B, H, lq))}
    a = {"out": np.zeros((B, lq, H, dv))}
    if grad_out is not None:
        g = np.where(rows[:, :, None, None], np.asarray(grad_out, dtype=np.float64), 0.0)
        r.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v), dlam=np.zeros(H))
        a.update({n: [np.zeros_like(r[n]) for _ in range(3)] for n in ("dq", "dk")})
        a.update(dv=np.zeros_like(v), dlam=np.zeros(H))
    for b in range(B):
        for h in range(H):
            c = h // G
            V = v[b, :, c]
            P, o = [], []
            for m in range(2):
                p, lse = _softmax(scale * (q[b, :, h, m] @ k[b, :, c, m].T), see[b])
                r["lse"][m, b, h] = lse
                P.append(p)
                o.append(p @ V)
                r["o"][m, b, :, h] = o[m]
            r["out"][b, :, h] = o[0] - lam[h] * o[1]
            a["out"][b, :, h] = (P[0] + abs(lam[h]) * P[1]) @ np.abs(V)
            if grad_out is None:
                continue
            gh = g[b, :, h]
            dp, dp_abs = gh @ V.T, np.abs(gh) @ np.abs(V).T
            r["dv"][b, :, c] += (P[0] - lam[h] * P[1]).T @ gh
            a["dv"][b, :, c] += (P[0] + abs(lam[h]) * P[1]).T @ np.abs(gh)
            r["dlam"][h] -= (P[1] * dp).sum()
            a["dlam"][h] += (P[1] * dp_abs).sum()
            for m in range(2):
                f = scale * (1.0 if m == 0 else -lam[h])
                D = (gh * o[m]).sum(axis=1, keepdims=True)
                D_abs = (np.abs(gh) * (P[m] @ np.abs(V))).sum(axis=1, keepdims=True)
                ds = f * P[m] * (dp - D)
                r["dq"][b, :, h, m] = ds @ k[b, :, c, m]
                r["dk"][b, :, c, m] += ds.T @ q[b, :, h, m]
                parts = (np.abs(ds), abs(f) * P[m] * D_abs, abs(f) * P[m] * dp_abs)
                for n, part in enumerate(parts):
                    a["dq"][n][b, :, h, m] = part @ np.abs(k[b, :, c, m])
                    a["dk"][n][b, :, c, m] += part.T @ np.abs(q[b, :, h, m])
    return r, a


def score_size(q, k, scale):
    """Largest sum of the absolute terms of a score, over the finite rows."""
    q, k = (np.nan_to_num(np.abs(np.asarray(x, dtype=np.float64)), nan=0.0, posinf=0.0) for x in (q, k))
    if q.size == 0 or k.size == 0:
        return 0.0
    return float(scale * np.linalg.norm(q, axis=-1).max() * np.linalg.norm(k, axis=-1).max())


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

def rotate(x, cos, sin, interleaved, inverse=False):
    """x: ... x H x d, cos and sin: ... x pairs (one row per token)."""
    x = np.array(x, dtype=np.float64)
    n = cos.shape[-1]
    c, s = cos[..., None, :], (-sin if inverse else sin)[..., None, :]
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    p, r = x[..., first].copy(), x[..., second].copy()
    x[..., first], x[..., second] = p * c - r * s, p * s + r * c
    return x


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------

def philox(counter, key):
    """Philox4x32-10 of one counter (four words) and key (two), in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        x, y = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(y >> 32) ^ c[1] ^ k[0], y & 0xFFFFFFFF, (x >> 32) ^ c[3] ^ k[1], x & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_factors(n, p, seed, offset, first=0):
    """What dropout multiplies elements first .. first + n - 1 by."""
    limit = int(np.rint(p * 65536))
    keep = 65536.0 / (65536 - limit) if limit < 65536 else 0.0
    m = np.empty(n)
    words, at = None, -1
    for e in range(first, first + n):
        if e >> 3 != at:
            at = e >> 3
            words = philox([at & 0xFFFFFFFF, at >> 32, offset & 0xFFFFFFFF, offset >> 32],
                           [seed & 0xFFFFFFFF, seed >> 32])
        u = words[(e & 7) >> 1] >> (16 * (e & 1)) & 0xFFFF
        m[e - first] = keep if u >= limit else 0.0
    return m


# ---------------------------------------------------------------------------
# norms, gate, residual scale
# ---------------------------------------------------------------------------

def _norm(t, layer, eps):
    t = t - t.mean(axis=1, keepdims=True) if layer else t
    rd = 1.0 / np.sqrt((t * t).mean(axis=1, keepdims=True) + eps)
    return t * rd, rd


def _norm_grad(dn, n, rd, layer):
    out = dn - n * (dn * n).mean(axis=1, keepdims=True)
    return (out - dn.mean(axis=1, keepdims=True) if layer else out) * rd


def norm_gate(x, z, w_post, b_post, gate, scale, w_pre, b_pre, layer, eps, m, grad_r=None, grad_h=None):
    """r, h and, with an upstream gradient, every gradient; ``m`` the factors of dropout or None.
    Returns (results, magnitudes) by name; absent arguments are None."""
    x = np.asarray(x, dtype=np.float64)
    n, c = x.shape
    one, zero = np.ones(c), np.zeros(c)
    wq, bq, sc, wp, bp = (np.asarray(t, dtype=np.float64) if t is not None else d for t, d in
                          ((w_post, one), (b_post, zero), (scale, one), (w_pre, one), (b_pre, zero)))
    gt = np.ones((1, c)) if gate is None else np.asarray(gate, dtype=np.float64)
    gr = np.repeat(gt, n // gt.shape[0], axis=0) if n else gt[:0]
    m = np.ones((n, c)) if m is None else m
    ab = np.abs
    res, mag = {}, {}
    r, r_abs = x, ab(x)
    if z is not None:
        z = np.asarray(z, dtype=np.float64)
        zn, zr = _norm(z, layer, eps)
        zn_abs = ab(zn) + ((ab(z) + ab(z).mean(axis=1, keepdims=True)) * zr if layer else 0.0)
        u, u_abs = zn * wq + bq, zn_abs * ab(wq) + ab(bq)
        r = x + m * sc * gr * u
        r_abs = r_abs + m * ab(sc) * ab(gr) * u_abs
        res["r"], mag["r"] = r, r_abs
    rn, rr = _norm(r, layer, eps)
    rn_abs = (r_abs + (r_abs.mean(axis=1, keepdims=True) if layer else 0.0)) * rr + ab(rn)
    res["h"], mag["h"] = rn * wp + bp, rn_abs * ab(wp) + ab(bp)
    if grad_r is None and grad_h is None:
        return res, mag

    def back(dn, t, rd, t_abs):  # magnitude of _norm_grad
        mean = lambda y: y.mean(axis=1, keepdims=True)  # noqa: E731
        return (dn + t_abs * mean(dn * t_abs) + (mean(dn) if layer else 0.0)) * rd

    dr, dr_abs = np.zeros((n, c)), np.zeros((n, c))
    if grad_r is not None:
        dr = np.asarray(grad_r, dtype=np.float64)
        dr_abs = ab(dr)
    if grad_h is not None:
        dh = np.asarray(grad_h, dtype=np.float64)
        dr = dr + _norm_grad(dh * wp, rn, rr, layer)
        dr_abs = dr_abs + back(ab(dh * wp), rn, rr, rn_abs)
        res["w_pre"], mag["w_pre"] = (dh * rn).sum(0), (ab(dh) * rn_abs).sum(0)
        res["b_pre"], mag["b_pre"] = dh.sum(0), ab(dh).sum(0)
    res["x"], mag["x"] = dr, dr_abs
    if z is not None:
        t, t_abs = dr * m, dr_abs * m
        du, du_abs = t * gr * sc, t_abs * ab(gr) * ab(sc)
        res["z"], mag["z"] = _norm_grad(du * wq, zn, zr, layer), back(du_abs * ab(wq), zn, zr, zn_abs)
        res["w_post"], mag["w_post"] = (du * zn).sum(0), (du_abs * zn_abs).sum(0)
        res["b_post"], mag["b_post"] = du.sum(0), du_abs.sum(0)
        res["scale"], mag["scale"] = (t * gr * u).sum(0), (t_abs * ab(gr) * u_abs).sum(0)
        if gate is not None:
            G = gt.shape[0]
            res["gate"] = (t * sc * u).reshape(G, -1, c).sum(1)
            mag["gate"] = (t_abs * ab(sc) * u_abs).reshape(G, -1, c).sum(1)
    return res, mag
