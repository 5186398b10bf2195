"""Pins of the oracle of the operators around an attention layer (oracle/attn.py):
closed forms, invariances, central differences of every gradient, the published
generator's known answers, and planted mistakes that the pins catch."""
import numpy as np
import pytest

from oracle import attn as A


def _inputs(seed, B=2, lq=5, lk=7, H=4, hk=2, d=3, dv=4):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((B, lq, H, 2, d)), rng.standard_normal((B, lk, hk, 2, d)),
            rng.standard_normal((B, lk, hk, dv)), rng.uniform(0.2, 0.8, H), rng.standard_normal((B, lq, H, dv)))


def test_one_key_gives_its_value():
    q, k, v, lam, _ = _inputs(1, lk=1)
    r, _ = A.attention(q, k, v, lam, 0.5, A.visible(2, 5, 1, False))
    want = (1 - lam)[None, None, :, None] * v[:, :, [0, 0, 1, 1]]
    assert np.allclose(r["out"], np.broadcast_to(want, r["out"].shape), atol=1e-14)


def test_equal_scores_average_the_seen_values():
    q, k, v, lam, _ = _inputs(2)
    mask = np.array([[1, 1, 0, 1, 0, 1, 1], [0, 1, 1, 1, 1, 1, 0]])
    see = A.visible(2, 5, 7, True, key_mask=mask, k_len=[7, 6], q_len=[5, 4])
    r, _ = A.attention(0 * q, k, v, lam, 0.5, see)
    for b, i in ((0, 0), (0, 4), (1, 2), (1, 4)):
        seen = v[b][see[b, i]]
        want = seen.mean(0) * (1 - lam[0]) if len(seen) else np.zeros((2, 4))
        assert np.allclose(r["out"][b, i, 0], want[0], atol=1e-14)
    assert not r["out"][1, 4].any()  # past q_len


def test_causal_rule_lets_the_last_query_see_everything():
    see = A.visible(1, 3, 5, True)[0]
    assert see.sum(1).tolist() == [3, 4, 5]
    assert A.visible(1, 5, 3, True)[0].sum(1).tolist() == [0, 0, 1, 2, 3]  # rows that see nothing
    assert A.visible(1, 4, 6, True, q_len=[3], k_len=[2])[0].sum(1).tolist() == [0, 1, 2, 0]


def test_hidden_keys_are_no_part_of_anything():
    q, k, v, lam, g = _inputs(3)
    mask = np.array([[1, 0, 1, 1, 1, 0, 1]] * 2)
    see = A.visible(2, 5, 7, False, key_mask=mask, k_len=[6, 5])
    r, _ = A.attention(q, k, v, lam, 0.5, see, g)
    k2, v2 = k.copy(), v.copy()
    k2[:, 1], v2[:, 1], k2[1, 5:], v2[0, 6] = np.nan, np.inf, np.inf, np.nan
    r2, _ = A.attention(q, k2, v2, lam, 0.5, see, g)
    for name in r:
        assert np.array_equal(r[name], r2[name]), name
    assert not r["dk"][:, 1].any() and not r["dv"][1, 5:].any()


@pytest.mark.parametrize("causal,plant", [(False, None), (True, None), (False, "no D"), (False, "lambda")])
def test_attention_gradients_against_differences(causal, plant):
    q, k, v, lam, g = _inputs(4)
    see = A.visible(2, 5, 7, causal, k_len=[7, 5], q_len=[5, 4])
    r, _ = A.attention(q, k, v, lam, 0.6, see, g)
    grads = [r["dq"], r["dk"], r["dv"], r["dlam"]]
    if plant == "no D":  # a softmax gradient without its mean term
        grads[0] = grads[0] + 0.6 * A.attention(q, k, v, lam, 0.6, see)[0]["o"][0].sum(-1)[..., None, None]
    if plant == "lambda":
        grads[3] = -grads[3]
    args, worst = [q, k, v, lam], 0.0
    for x, dx in zip(args, grads):
        flat = x.reshape(-1)
        for e in range(0, flat.size, max(1, flat.size // 23)):
            keep, side = flat[e], []
            for s in (1e-5, -1e-5):
                flat[e] = keep + s
                side.append((A.attention(*args, 0.6, see)[0]["out"] * g).sum())
            flat[e] = keep
            worst = max(worst, abs((side[0] - side[1]) / 2e-5 - dx.reshape(-1)[e]))
    assert (worst < 1e-8) == (plant is None), worst


def test_rotation_keeps_lengths_and_turns_back():
    rng = np.random.default_rng(5)
    x, ang = rng.standard_normal((3, 4, 10)), rng.standard_normal((3, 4))
    for inter in (False, True):
        y = A.rotate(x, np.cos(ang), np.sin(ang), inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        assert np.array_equal(y[..., 8:], x[..., 8:])
        assert np.allclose(A.rotate(y, np.cos(ang), np.sin(ang), inter, inverse=True), x, atol=1e-14)
    # the product of two turned heads depends on the difference of their angles alone
    a, b = rng.standard_normal(8), rng.standard_normal(8)
    f = rng.standard_normal(4)
    dot = [A.rotate(a[None], np.cos((t + 3) * f), np.sin((t + 3) * f), True)[0]
           @ A.rotate(b[None], np.cos(t * f), np.sin(t * f), True)[0] for t in (0.0, 7.0)]
    assert abs(dot[0] - dot[1]) < 1e-12


def test_generator_known_answers():
    """The known answers that the generator's authors publish with it (counter, key -> words)."""
    assert A.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert A.philox([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_dropout_factors_keep_the_mean():
    m = A.dropout_factors(40000, 0.3, 12345, 3)
    assert abs(m.mean() - 1.0) < 5 * np.sqrt(0.3 / 0.7 / 40000)
    assert np.array_equal(A.dropout_factors(100, 0.3, 12345, 3, first=777), m[777:877])
    assert not A.dropout_factors(20, 1.0, 1, 1).any() and (A.dropout_factors(20, 0.0, 1, 1) == 1).all()


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_norm_gradients_against_differences(layer, gated):
    rng = np.random.default_rng(6)
    n, c = 6, 5
    arg = {"x": rng.standard_normal((n, c)), "z": rng.standard_normal((n, c)), "w_post": rng.standard_normal(c),
           "b_post": rng.standard_normal(c), "gate": rng.standard_normal((3, c)) if gated else None,
           "scale": rng.standard_normal(c), "w_pre": rng.standard_normal(c), "b_pre": rng.standard_normal(c)}
    m = A.dropout_factors(n * c, 0.25, 9, 9).reshape(n, c)
    gr, gh = rng.standard_normal((n, c)), rng.standard_normal((n, c))

    def loss():
        r, _ = A.norm_gate(**arg, layer=layer, eps=1e-3, m=m)
        return (r["r"] * gr).sum() + (r["h"] * gh).sum()

    res, mag = A.norm_gate(**arg, layer=layer, eps=1e-3, m=m, grad_r=gr, grad_h=gh)
    for name, x in arg.items():
        if x is None:
            continue
        flat = x.reshape(-1)
        for e in range(flat.size):
            keep, side = flat[e], []
            for s in (1e-5, -1e-5):
                flat[e] = keep + s
                side.append(loss())
            flat[e] = keep
            assert abs((side[0] - side[1]) / 2e-5 - res[name].reshape(-1)[e]) < 1e-7, name
        assert (np.abs(res[name]) <= mag[name] + 1e-12).all(), name
