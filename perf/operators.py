"""Performance cases of the operators around an exact attention layer:
differential attention, rotary positions, the norms before and after a block
with its gate and residual scale, and dropout.

A case is one use of the public entry points of ``paper_1907_00641_amd`` at
one size; ``listed()`` holds the named ones, ``draw(rng)`` gives further ones
of the same ranges.  ``prepare`` makes the inputs on the GPU from the seed
alone, ``run`` is one pass (``own``: through the framework's kernels, else in
plain torch operations in 32 bits), ``work`` the traffic and arithmetic that
a pass cannot do without, ``exact`` the same results in 64 bits from the
operators' definitions.

Kinds of case:

* ``attn``    differential attention, ``train``: forward and the gradients of
              q, k, v and lambda; else the forward pass alone (with one query
              per sequence: a decoding step over a cache)
* ``rotary``  rotation of q and k, ``train``: and of their gradients back
* ``norm``    r = x + drop(scale gate N(z)), h = N(r); ``train``: and every
              gradient
* ``dropout`` values forward, their gradients with the same mask

Queries and keys are i.i.d. normal, scaled so that the scores have a standard
deviation of 1.5; values, activations and upstream gradients are N(0, 1).
"""
import functools
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _attn(name, batch, lq, lk, heads, kv_heads, d, dtype, train=False, causal=False, ragged=False, masked=False):
    case = {"kind": "attn", "batch": batch, "lq": lq, "lk": lk, "heads": heads, "kv_heads": kv_heads, "d": d,
            "dtype": dtype, "train": train, "causal": causal, "ragged": ragged, "masked": masked}
    return dict(case, name=name) if name else case


def _rotary(name, batch, length, heads, kv_heads, d, rot, dtype, interleaved=False, train=False, start=0):
    case = {"kind": "rotary", "batch": batch, "length": length, "heads": heads, "kv_heads": kv_heads, "d": d,
            "rot": rot, "dtype": dtype, "interleaved": interleaved, "train": train, "start": start}
    return dict(case, name=name) if name else case


def _norm(name, samples, rows, channels, dtype, norm="rms", train=False, p=0.0, gated=True):
    case = {"kind": "norm", "samples": samples, "rows": rows, "channels": channels, "dtype": dtype, "norm": norm,
            "train": train, "p": p, "gated": gated}
    return dict(case, name=name) if name else case


def _dropout(name, rows, channels, dtype, p):
    case = {"kind": "dropout", "rows": rows, "channels": channels, "dtype": dtype, "p": p}
    return dict(case, name=name) if name else case


def listed():
    return [
        # smallest: one new token of one sequence over a short cache, where latency is all
        _attn("decode 1x300 h4 d32 bf16", 1, 1, 300, 4, 4, 32, "bf16"),
        # a decoding step of eight sequences of different lengths, 32 query heads on 8 key heads, a long cache
        _attn("decode 8x16384 h32/8 d64 bf16", 8, 1, 16384, 32, 8, 64, "bf16", ragged=True),
        # training on the 20x20x12 feature map of two 160x160x96 patches
        _attn("train 2x4800 h8 d64 bf16", 2, 4800, 4800, 8, 8, 64, "bf16", train=True),
        # training on ragged sequences with hidden keys, shared heads, a head size that is no power of two
        _attn("train 3x1001 h6/2 d40 f16", 3, 1001, 1001, 6, 2, 40, "f16", train=True, causal=True, ragged=True,
              masked=True),
        # training in the framework's own type on a 13x13x13 map
        _attn("train 1x2197 h4 d32 f32", 1, 2197, 2197, 4, 4, 32, "f32", train=True),
        # largest: training on one long causal sequence
        _attn("train 1x16384 h8/2 d64 bf16", 1, 16384, 16384, 8, 2, 64, "bf16", train=True, causal=True),
        # a block's norms for the tokens of one decoding step
        _norm("norm 8x1024 bf16", 8, 1, 1024, "bf16"),
        # training on the 40x40x24 map, gated per sample, with dropout
        _norm("norm train 2x38400x512 bf16", 2, 38400, 512, "bf16", train=True, p=0.1),
        # dropout on the same activations, and on a small ragged set in 32 bits
        _dropout("dropout 76800x512 bf16", 76800, 512, "bf16", 0.1),
        _dropout("dropout 2197x75 f32", 2197, 75, "f32", 0.25),
        # positions of the two patches' queries and keys, in training
        _rotary("rotary train 2x4800 h8 d64 bf16", 2, 4800, 8, 8, 64, 64, "bf16", train=True),
        # part of the head, interleaved, shared heads, far into a long context
        _rotary("rotary 1x16384 h32/8 d128 f16", 1, 16384, 32, 8, 128, 64, "f16", interleaved=True, start=100000),
    ]


def _spread(rng, lo, hi):
    """A whole number spread over [lo, hi] by its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    case = _drawn(rng)
    while 3072 in case.values():  # a size that stands for nothing here
        case = _drawn(rng)
    return case


def _drawn(rng):
    kind = rng.choice(["decode", "prefill", "attn", "attn", "attn", "norm", "norm", "dropout", "rotary"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("decode", "prefill", "attn"):
        kv_heads = rng.choice([1, 2, 4, 5, 8])
        group = rng.choice([1, 1, 2, 4, 7]) if kind != "decode" else rng.choice([1, 2, 4, 8])
        d = rng.choice([16, 32, 40, 64, 64, 64, 128]) if dtype != "f32" else rng.choice([16, 20, 32, 64])
        ragged = rng.random() < 0.5
        if kind == "decode":
            batch = rng.choice([1, 1, 2, 5, 8, 16])
            lk = _spread(rng, 16, min(40000, 100000000 // (batch * kv_heads * d)))
            return _attn(None, batch, rng.choice([1, 1, 1, 3]), lk, kv_heads * group, kv_heads, d, dtype,
                         causal=True, ragged=ragged)
        batch = rng.choice([1, 1, 2, 3])
        pairs = 1.0e9 * 64 / max(d, 32) / (batch * kv_heads * group) / (8 if dtype == "f32" else 1)
        lq = _spread(rng, 24, min(9000, math.isqrt(int(pairs))))
        lk = lq if rng.random() < 0.7 else _spread(rng, 24, min(9000, int(pairs) // lq))
        return _attn(None, batch, lq, lk, kv_heads * group, kv_heads, d, dtype, train=kind == "attn",
                     causal=rng.random() < 0.5 and lk >= lq, ragged=ragged, masked=rng.random() < 0.2)
    if kind == "rotary":
        d = rng.choice([32, 64, 64, 80, 128])
        heads = rng.choice([4, 8, 16, 32])
        return _rotary(None, rng.choice([1, 2, 3]), _spread(rng, 1, 65536 * 32 // (heads * d)), heads,
                       max(1, heads // rng.choice([1, 4])), d, rng.choice([d, d // 2, 8 * (d // 16)]), dtype,
                       rng.random() < 0.5, rng.random() < 0.5, rng.choice([0, 0, 1000, 50000]))
    if kind == "norm":
        channels = rng.choice([_spread(rng, 16, 8192), 64 * _spread(rng, 1, 128)])
        samples = rng.choice([1, 2, 8])
        rows = _spread(rng, 1, max(2, 30000000 // (channels * samples)))
        return _norm(None, samples, rows, channels, dtype, rng.choice(["rms", "rms", "layer"]), rng.random() < 0.6,
                     rng.choice([0.0, 0.1, 0.3]), rng.random() < 0.7)
    channels = _spread(rng, 8, 2048)
    return _dropout(None, _spread(rng, 16, 39000000 // channels), channels, dtype, rng.choice([0.05, 0.1, 0.5]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, times=1.0, dtype=dt):
        return (times * torch.randn(*shape, generator=gen, device=dev)).to(dtype)

    st = {"case": case}
    if case["kind"] == "attn":
        B, H, Hk, d, lq, lk = (case[x] for x in ("batch", "heads", "kv_heads", "d", "lq", "lk"))
        st["q"] = normal(B, lq, H, 2, d, times=1.5)
        st["k"] = normal(B, lk, Hk, 2, d)
        st["v"] = normal(B, lk, Hk, 2 * d)
        st["lam"] = (0.2 + 0.6 * torch.rand(H, generator=gen, device=dev)).to(dt)
        if case["train"]:
            st["dout"] = normal(B, lq, H, 2 * d)
        st["q_len"] = st["k_len"] = st["key_mask"] = None
        if case["ragged"]:  # one sequence of full length, the others shorter
            part = 0.5 + 0.5 * torch.rand(B, generator=gen, device=dev)
            part[0] = 1.0
            st["k_len"] = (part * lk).to(torch.int32).clamp(min=1)
            if lq == lk:
                st["q_len"] = st["k_len"]
        if case["masked"]:
            st["key_mask"] = torch.rand(B, lk, generator=gen, device=dev) >= 0.2
    elif case["kind"] == "rotary":
        B, n, H, Hk, d, rot = (case[x] for x in ("batch", "length", "heads", "kv_heads", "d", "rot"))
        st["q"], st["k"] = normal(B, n, H, d), normal(B, n, Hk, d)
        if case["train"]:
            st["dq"], st["dk"] = normal(B, n, H, d), normal(B, n, Hk, d)
        # the table a model keeps: cosine and sine of every position's angles
        freq = 10000.0 ** (-torch.arange(0, rot, 2, device=dev, dtype=torch.float64) / rot)
        angle = torch.arange(case["start"] + n, device=dev, dtype=torch.float64)[:, None] * freq
        st["table"] = torch.stack([torch.cos(angle), torch.sin(angle)], 2).float().contiguous()
        st["pos"] = torch.randint(case["start"], case["start"] + n, (B, n), generator=gen, device=dev,
                                  dtype=torch.int32)
    elif case["kind"] == "norm":
        n, c = case["samples"] * case["rows"], case["channels"]
        st["x"], st["z"] = normal(n, c, times=2.0), normal(n, c)
        f32 = torch.float32
        st["w_post"], st["w_pre"] = 1 + normal(c, times=0.1, dtype=f32), 1 + normal(c, times=0.1, dtype=f32)
        layer = case["norm"] == "layer"
        st["b_post"] = normal(c, times=0.1, dtype=f32) if layer else None
        st["b_pre"] = normal(c, times=0.1, dtype=f32) if layer else None
        st["scale"] = 0.3 + normal(c, times=0.1, dtype=f32)
        st["gate"] = normal(case["samples"], c) if case["gated"] else None
        if case["train"]:
            st["dr"], st["dh"] = normal(n, c), normal(n, c)
        st["seed"], st["offset"] = seed, 7
    else:
        n, c = case["rows"], case["channels"]
        st["x"], st["dy"] = normal(n, c), normal(n, c)
        st["seed"], st["offset"] = seed, 11
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"attn": _own_attn, "rotary": _own_rotary, "norm": _own_norm, "dropout": _own_dropout}[kind](st)
    return {"attn": _plain_attn, "rotary": _plain_rotary, "norm": _plain_norm, "dropout": _plain_dropout}[kind](st)


def _own_attn(st):
    import paper_1907_00641_amd as P

    case = st["case"]
    how = dict(causal=case["causal"], q_len=st["q_len"], k_len=st["k_len"], key_mask=st["key_mask"])
    q, k, v, lam = st["q"], st["k"], st["v"], st["lam"]
    if not case["train"]:
        return P.pam_diff_attn_fwd(q, k, v, lam, **how)
    out, saved = P.pam_diff_attn_fwd(q, k, v, lam, save=True, **how)
    return (out,) + tuple(P.pam_diff_attn_bwd(q, k, v, lam, saved, st["dout"], **how))


def _own_rotary(st):
    import paper_1907_00641_amd as P

    how = dict(pos=st["pos"], interleaved=st["case"]["interleaved"])
    res = tuple(P.pam_rotary(st["q"], st["k"], st["table"], **how))
    if st["case"]["train"]:
        res += tuple(P.pam_rotary(st["dq"], st["dk"], st["table"], inverse=True, **how))
    return res


def _own_norm(st):
    import paper_1907_00641_amd as P

    case = st["case"]
    how = dict(z=st["z"], w_post=st["w_post"], b_post=st["b_post"], gate=st["gate"], scale=st["scale"],
               w_pre=st["w_pre"], b_pre=st["b_pre"], norm=case["norm"], p=case["p"], seed=st["seed"],
               offset=st["offset"])
    res = list(P.pam_norm_gate_fwd(st["x"], **how))
    if case["train"]:
        grads = P.pam_norm_gate_bwd(st["x"], grad_r=st["dr"], grad_h=st["dh"], **how)
        res += [grads[name] for name in _norm_grads(case)]
    return res


def _own_dropout(st):
    import paper_1907_00641_amd as P

    how = (st["case"]["p"], st["seed"], st["offset"])
    return P.pam_dropout(st["x"], *how), P.pam_dropout(st["dy"], *how)


def _norm_grads(case):
    names = ["x", "z", "w_post", "scale", "w_pre"]
    return names + (["gate"] if case["gated"] else []) + (["b_post", "b_pre"] if case["norm"] == "layer" else [])


def _visible(st):
    """Which key each query may see (batch x lq x lk), or None where every one is."""
    case = st["case"]
    B, lq, lk = case["batch"], case["lq"], case["lk"]
    dev = st["q"].device
    if not case["causal"] and st["k_len"] is None and st["q_len"] is None and st["key_mask"] is None:
        return None
    i, j = torch.arange(lq, device=dev)[None, :, None], torch.arange(lk, device=dev)[None, None, :]
    k_len = torch.full((B,), lk, device=dev) if st["k_len"] is None else st["k_len"].long()
    q_len = torch.full((B,), lq, device=dev) if st["q_len"] is None else st["q_len"].long()
    k_len, q_len = k_len[:, None, None], q_len[:, None, None]
    see = (j < k_len) & (i < q_len)
    if case["causal"]:
        see = see & (j <= i + k_len - q_len)
    if st["key_mask"] is not None:
        see = see & st["key_mask"][:, None, :]
    return see


def _plain_attn(st):
    case = st["case"]
    B, H, Hk, d, lq, lk = (case[x] for x in ("batch", "heads", "kv_heads", "d", "lq", "lk"))
    G, dt, scale = H // Hk, st["q"].dtype, 1.0 / math.sqrt(d)
    # heads first: q is (B, Hk, G, 2, lq, d), k is (B, Hk, 1, 2, lk, d), v is (B, Hk, 1, lk, 2 d)
    q = st["q"].float().reshape(B, lq, Hk, G, 2, d).permute(0, 2, 3, 4, 1, 5).contiguous()
    k = st["k"].float().permute(0, 2, 3, 1, 4).contiguous().unsqueeze(2)
    v = st["v"].float().permute(0, 2, 1, 3).contiguous().unsqueeze(2)
    lam = st["lam"].float().reshape(1, Hk, G, 1, 1)
    see = _visible(st)
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    if see is not None:
        see = see[:, None, None, None]
        s = torch.where(see, s, -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3.0e38)
    p = torch.exp(s - top)
    del s
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-37)
    w = p[:, :, :, 0] - lam * p[:, :, :, 1]
    out = torch.matmul(w, v)
    out_t = out.permute(0, 3, 1, 2, 4).reshape(B, lq, H, 2 * d).to(dt)
    if not case["train"]:
        return out_t
    do = st["dout"].float().reshape(B, lq, Hk, G, 2 * d).permute(0, 2, 3, 1, 4).contiguous()
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    dlam = -(p[:, :, :, 1] * dp).sum(dim=(0, 3, 4)).reshape(H)
    dv = torch.matmul(w.transpose(-1, -2).contiguous(), do).sum(2)
    del w
    dp = dp.unsqueeze(3)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    del p, dp
    sign = torch.stack([torch.ones_like(lam), -lam], 3)
    ds = ds * sign
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q).sum(2)
    dq = dq.permute(0, 4, 1, 2, 3, 5).reshape(B, lq, H, 2, d)
    dk = dk.permute(0, 3, 1, 2, 4)
    dv = dv.permute(0, 2, 1, 3)
    return out_t, dq.to(dt), dk.to(dt).contiguous(), dv.to(dt).contiguous(), dlam.to(dt)


def _rotate(x, table, rot, interleaved, sign):
    c, s = table[:, :, None, :, 0], sign * table[:, :, None, :, 1]
    y = x.float()
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    else:
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _plain_rotary(st):
    case = st["case"]
    t = st["table"][st["pos"].long()]
    how = (t, case["rot"], case["interleaved"])
    res = (_rotate(st["q"], *how, 1.0), _rotate(st["k"], *how, 1.0))
    if case["train"]:
        res += (_rotate(st["dq"], *how, -1.0), _rotate(st["dk"], *how, -1.0))
    return res


def _philox_round(state, _):
    """One round of the counter-based generator Philox4x32 on 32-bit words held in 64 bits."""
    (a, b, c, d), (k0, k1) = state
    low = 0xFFFFFFFF
    x, y = a * 0xD2511F53, c * 0xCD9E8D57
    words = (((y >> 32) & low) ^ b ^ k0, y & low, ((x >> 32) & low) ^ d ^ k1, x & low)
    return words, ((k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low)


def _kept(n, p, seed, offset, dev):
    """What dropout multiplies n values by: eight values take the eight 16-bit numbers of one counter."""
    low = 0xFFFFFFFF
    at = torch.arange((n + 7) // 8, device=dev)
    words = (at & low, at >> 32, torch.full_like(at, offset & low), torch.full_like(at, offset >> 32))
    words, _ = functools.reduce(_philox_round, range(10), (words, (seed & low, seed >> 32)))
    words = torch.stack(words, 1)
    u = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n]
    limit = round(p * 65536)
    return (u >= limit).float() * (65536.0 / (65536 - limit))


def _plain_dropout(st):
    case, x, dy = st["case"], st["x"], st["dy"]
    m = _kept(x.numel(), case["p"], st["seed"], st["offset"], x.device).reshape(x.shape)
    return (x.float() * m).to(x.dtype), (dy.float() * m).to(x.dtype)


def _normed(x, layer, eps=1e-6):
    """Normalised rows and their reciprocal deviation."""
    if layer:
        x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + eps)
    return x * r, r


def _normed_grad(dn, n, r, layer):
    """Gradient of the rows that were normalised to n with deviation 1 / r."""
    dx = dn - n * (dn * n).mean(1, keepdim=True)
    if layer:
        dx = dx - dn.mean(1, keepdim=True)
    return dx * r


def _plain_norm(st):
    case = st["case"]
    layer, dt, S = case["norm"] == "layer", st["x"].dtype, case["samples"]
    n, c = st["x"].shape
    zn, zr = _normed(st["z"].float(), layer)
    u = zn * st["w_post"]
    if layer:
        u = u + st["b_post"]
    gate = st["gate"].float().repeat_interleave(case["rows"], 0) if case["gated"] else torch.ones_like(u)
    m = _kept(n * c, case["p"], st["seed"], st["offset"], u.device).reshape(n, c) if case["p"] else 1.0
    r = st["x"].float() + st["scale"] * gate * u * m
    rn, rr = _normed(r, layer)
    h = rn * st["w_pre"]
    if layer:
        h = h + st["b_pre"]
    res = [r.to(dt), h.to(dt)]
    if not case["train"]:
        return res
    dh = st["dh"].float()
    dr = st["dr"].float() + _normed_grad(dh * st["w_pre"], rn, rr, layer)
    t = dr * m
    du = t * gate * st["scale"]
    g = {"x": dr.to(dt), "z": _normed_grad(du * st["w_post"], zn, zr, layer).to(dt), "w_post": (du * zn).sum(0),
         "scale": (t * gate * u).sum(0), "w_pre": (dh * rn).sum(0), "b_post": du.sum(0), "b_pre": dh.sum(0)}
    if case["gated"]:
        g["gate"] = (t * st["scale"] * u).reshape(S, case["rows"], c).sum(1).to(dt)
    return res + [g[name] for name in _norm_grads(case)]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _lengths(case):
    """Average visible keys of a query, and the share of the tokens that ragged batches hold."""
    part = 1.0 if not case["ragged"] else (1.0 + 0.75 * (case["batch"] - 1)) / case["batch"]
    lk = case["lk"] * part
    keys = lk
    if case["causal"]:
        lq = case["lq"] * (part if case["lq"] == case["lk"] else 1.0)
        keys = lk - (lq - 1) / 2
    return keys * (0.8 if case["masked"] else 1.0), part


def work(case):
    e = BYTES[case["dtype"]]
    if case["kind"] == "attn":
        B, H, Hk, d, lq, lk = (case[x] for x in ("batch", "heads", "kv_heads", "d", "lq", "lk"))
        keys, part = _lengths(case)
        rows = B * lq * (part if lq == lk else 1.0)
        q, kv = rows * H * 2 * d * e, B * lk * part * Hk * 2 * d * e
        pair = rows * H * keys * 2 * 2 * d  # one product of a head's pairs with 2 d channels
        if case["train"]:  # q, k, v, dout in, out and four gradients out; scores, out, dp, dv, dq, dk
            return {"bytes": 4 * q + 4 * kv, "flops": 6 * pair}
        return {"bytes": 2 * q + 2 * kv, "flops": 2 * pair}  # scores, and the two maps' difference times v
    if case["kind"] == "rotary":
        n = case["batch"] * case["length"]
        moved = n * (case["heads"] + case["kv_heads"]) * case["d"] * e * 2 + case["length"] * case["rot"] * 4 + n * 4
        times = 2 if case["train"] else 1
        return {"bytes": times * moved, "flops": times * n * (case["heads"] + case["kv_heads"]) * case["rot"] * 3}
    if case["kind"] == "norm":
        n = case["samples"] * case["rows"] * case["channels"]
        return {"bytes": n * e * (8 if case["train"] else 4), "flops": n * (50 if case["train"] else 15)}
    n = case["rows"] * case["channels"]
    return {"bytes": 4 * n * e, "flops": 4 * n}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    return {"attn": _exact_attn, "rotary": _exact_rotary, "norm": _exact_norm, "dropout": _exact_dropout}[kind](case, st)


def _exact_head(case, st, b, h, hk):
    """Output and, in training, gradients of one head of one sequence, by differentiation."""
    x = [t.double().requires_grad_(case["train"]) for t in
         (st["q"][b, :, h], st["k"][b, :, hk], st["v"][b, :, hk], st["lam"][h])]
    q, k, v, lam = x
    lq, lk, d = case["lq"], case["lk"], case["d"]
    nk = lk if st["k_len"] is None else int(st["k_len"][b])
    nq = lq if st["q_len"] is None else int(st["q_len"][b])
    allowed = torch.zeros(lq, lk, dtype=torch.bool, device=q.device)
    allowed[:nq, :nk] = True
    if case["causal"]:
        allowed &= torch.ones_like(allowed).tril(nk - nq)
    if st["key_mask"] is not None:
        allowed &= st["key_mask"][b]
    rows = allowed.any(1, keepdim=True)

    def attend(m):
        s = (q[:, m] @ k[:, m].t()) / math.sqrt(d)
        s = s.masked_fill(rows & ~allowed, -math.inf)
        return (torch.softmax(s, 1) * rows) @ v

    out = attend(0) - lam * attend(1)
    if not case["train"]:
        return (out,)
    return (out.detach(),) + torch.autograd.grad(out, x, st["dout"][b, :, h].double())


def _exact_attn(case, st):
    B, H, Hk = case["batch"], case["heads"], case["kv_heads"]
    f64 = dict(dtype=torch.float64)
    out = torch.zeros(B, case["lq"], H, 2 * case["d"], device=st["q"].device, **f64)
    dq, dk, dv, dlam = (torch.zeros_like(st[x], **f64) for x in ("q", "k", "v", "lam"))
    for b in range(B):
        for h in range(H):
            r = _exact_head(case, st, b, h, h // (H // Hk))
            out[b, :, h] = r[0]
            if case["train"]:
                dq[b, :, h] += r[1]
                dk[b, :, h // (H // Hk)] += r[2]
                dv[b, :, h // (H // Hk)] += r[3]
                dlam[h] += r[4]
    return (out, dq, dk, dv, dlam) if case["train"] else out


def _exact_rotary(case, st):
    half = case["rot"] // 2
    turn = torch.view_as_complex(st["table"].double())[st["pos"].long()].unsqueeze(2)

    def rotated(x, w):
        y = x.double()
        part = y[..., : 2 * half]
        if case["interleaved"]:
            z = torch.view_as_complex(part.unflatten(-1, (half, 2)).contiguous()) * w
            y[..., : 2 * half] = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(part[..., :half].contiguous(), part[..., half:].contiguous()) * w
            y[..., : 2 * half] = torch.cat([z.real, z.imag], -1)
        return y

    res = (rotated(st["q"], turn), rotated(st["k"], turn))
    return res + (rotated(st["dq"], turn.conj()), rotated(st["dk"], turn.conj())) if case["train"] else res


def _exact_kept(n, p, seed, offset):
    """The factors of dropout, with the generator written on numpy's 64-bit words."""
    u = np.uint64
    low, s32 = u(0xFFFFFFFF), u(32)
    ctr = np.zeros((4, (n + 7) // 8), dtype=np.uint64)
    ctr[0] = np.arange(ctr.shape[1], dtype=np.uint64) & low
    ctr[1] = np.arange(ctr.shape[1], dtype=np.uint64) >> s32
    ctr[2], ctr[3] = offset & 0xFFFFFFFF, offset >> 32
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = np.stack([(p1 >> s32) ^ ctr[1] ^ u(key[0]), p1 & low, (p0 >> s32) ^ ctr[3] ^ u(key[1]), p0 & low])
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    parts = ctr.T.astype("<u4").copy().view("<u2").reshape(-1)[:n]
    limit = round(p * 65536)
    return torch.from_numpy(np.where(parts >= limit, 65536.0 / (65536 - limit), 0.0))


def _exact_dropout(case, st):
    x = st["x"]
    m = _exact_kept(x.numel(), case["p"], st["seed"], st["offset"]).reshape(x.shape).to(x.device)
    return x.double() * m, st["dy"].double() * m


def _exact_norm(case, st):
    n, c = st["x"].shape
    names = [x for x in ["x", "z", "w_post", "scale", "w_pre", "gate", "b_post", "b_pre"] if st[x] is not None]
    v = {x: st[x].double().requires_grad_(case["train"]) for x in names}

    def norm(t, w, b):
        if case["norm"] == "layer":
            return torch.nn.functional.layer_norm(t, (c,), v[w], v[b], 1e-6)
        return t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) * v[w]

    y = norm(v["z"], "w_post", "b_post") * v["scale"]
    if case["gated"]:
        y = (y.reshape(case["samples"], case["rows"], c) * v["gate"][:, None]).reshape(n, c)
    if case["p"]:
        y = y * _exact_kept(n * c, case["p"], st["seed"], st["offset"]).reshape(n, c).to(y.device)
    r = v["x"] + y
    h = norm(r, "w_pre", "b_pre")
    res = [r.detach(), h.detach()]
    if case["train"]:
        order = _norm_grads(case)
        res += torch.autograd.grad([r, h], [v[x] for x in order], [st["dr"].double(), st["dh"].double()])
    return res
