"""The 64-bit oracle of attention over packed sequences and from a paged cache (oracle/packed.py) against
differentiation and against torch's own 8-bit type (no GPU needed)."""
import math

import numpy as np
import pytest
import torch

from oracle import packed as O


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradients(causal):
    rng = np.random.default_rng(1)
    q_ends, k_ends = [1, 1, 8, 12], [0, 3, 9, 18]
    q, k, v, g = (rng.standard_normal(s) for s in ((13, 4, 5), (19, 2, 5), (19, 2, 6), (13, 4, 6)))
    r, a = O.packed(q, k, v, 0.4, q_ends, k_ends, causal, g)
    t = [torch.from_numpy(x).requires_grad_() for x in (q, k, v)]
    out = torch.zeros(13, 4, 6, dtype=torch.float64)
    for b in range(3):
        x, y = slice(q_ends[b], q_ends[b + 1]), slice(k_ends[b], k_ends[b + 1])
        n, m = x.stop - x.start, y.stop - y.start
        for h in range(4):
            s = 0.4 * t[0][x, h] @ t[1][y, h // 2].t()
            see = torch.ones(n, m, dtype=torch.bool)
            if causal:
                see = see.tril(m - n)
            rows = see.any(1, keepdim=True)  # a row of -inf has no gradient but NaN
            p = torch.softmax(s.masked_fill(rows & ~see, -math.inf), 1) * rows
            out[x, h] = p @ t[2][y, h // 2]
    want = [out.detach()] + list(torch.autograd.grad(out, t, torch.from_numpy(g)))
    for name, w in zip(("out", "dq", "dk", "dv"), want):
        assert np.allclose(r[name], w.numpy(), atol=1e-12), name
        top = a[name] if name in ("out", "dv") else a[name][1] + a[name][2]
        assert (np.abs(r[name]) <= top + 1e-12).all(), name


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
def test_head_norm_gradients(layer, interleaved, per_head):
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((2, 3, 4, 10)), rng.standard_normal((2, 3, 4, 10))
    w = rng.standard_normal((4, 10) if per_head else 10)
    angle = rng.uniform(-3, 3, (2, 3, 4))
    r, a = O.head_norm(x, w, np.cos(angle), np.sin(angle), layer, 1e-3, interleaved, g)
    tx, tw = torch.from_numpy(x).requires_grad_(), torch.from_numpy(w).requires_grad_()
    z = tx - tx.mean(-1, keepdim=True) if layer else tx
    y = z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-3) * tw
    part = y[..., :8]
    pair = part.unflatten(-1, (4, 2)) if interleaved else torch.stack([part[..., :4], part[..., 4:]], -1)
    turned = torch.view_as_complex(pair.contiguous()) * torch.polar(torch.ones(2, 3, 4, dtype=torch.float64),
                                                                    torch.from_numpy(angle))[:, :, None]
    turned = torch.view_as_real(turned)
    turned = turned.flatten(-2) if interleaved else torch.cat([turned[..., 0], turned[..., 1]], -1)
    y = torch.cat([turned, y[..., 8:]], -1)
    gx, gw = torch.autograd.grad(y, (tx, tw), torch.from_numpy(g))
    for name, want in (("y", y.detach()), ("dx", gx), ("dw", gw)):
        assert np.allclose(r[name], want.numpy(), atol=1e-12), name
        assert (np.abs(r[name]) <= a[name] + 1e-12).all(), name


def test_stored_rows():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((200, 16)) * np.exp2(rng.uniform(-20, 20, (200, 1)))).astype(np.float32)
    x[0], x[1] = 0.0, 1e-42
    top = torch.tensor(448.0)
    t = torch.from_numpy(x)
    scale = (t.abs().amax(-1) / top).clamp(min=2.0 ** -126)
    want = (t / scale[:, None]).to(torch.float8_e4m3fn).double().numpy()
    y, s = O.stored(x, "e4m3")
    assert np.array_equal(s, scale.numpy()) and np.array_equal(y, want)
    y, s = O.stored(x, "int8")
    assert np.abs(y).max() == 127 and (np.abs(y * s[:, None] - x) <= 0.5001 * s[:, None]).all()
    x[5, 3], x[6, 0] = np.inf, np.nan
    _, s = O.stored(x, "int8")
    assert np.isnan(s[[5, 6]]).all() and np.isfinite(np.delete(s, [5, 6])).all()
