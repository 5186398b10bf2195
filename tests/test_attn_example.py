"""The example layer of the attention layer's operators: its training step and its token-by-token form."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import examples.attention_layer as E

    return E


def test_training_lowers_the_loss(example):
    import torch

    for dtype in (torch.float32, torch.bfloat16):
        losses = example.train(steps=12, p=0.0, dtype=dtype)
        assert np.isfinite(losses).all() and losses[-1] < 0.9 * losses[0], losses


def test_gradients_against_differences(example):
    """loss(w + e dw) - loss(w - e dw) over 2 e, in fp32.  The loss is a mean of 10^4 products of magnitude 1, each off
    by less than 1e-5 and at random: 1e-7; the difference quotient with e = 1e-2 is off by that over e, 1e-5, and by the
    third derivative times e^2 / 6: 2 % of the larger of itself and 0.01 covers both."""
    import torch

    side, b, c = 6, 2, 48
    layer = example.Layer(c, 4, 2, 16, torch.float32, seed=3)
    table = example.voxel_table(side, 16)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    x, gate, up = normal(b, side ** 3, c), normal(b, c), normal(b, side ** 3, c)

    def loss(causal):
        return (layer.forward(x, table, gate, p=0.2, seed=9, causal=causal)[0].double() * up.double()).mean().item()

    for causal in (False, True):
        _, kept = layer.forward(x, table, gate, p=0.2, seed=9, causal=causal)
        grads = layer.backward(kept, up / up.numel())
        for name in [*layer.w, "x", "gate"]:
            at = {"x": x, "gate": gate}.get(name, layer.w.get(name))
            g = grads[name].double()
            # along the gradient's sign, so that the difference is not lost in rounding
            step = (g.sign() * normal(*at.shape).abs().double()).float() * at.abs().mean()
            want, keep, e = float((g * step.double()).sum()), at.clone(), 1e-2
            at.copy_(keep + e * step)
            above = loss(causal)
            at.copy_(keep - e * step)
            below = loss(causal)
            at.copy_(keep)
            got = (above - below) / (2 * e)
            print(f"  {name} causal={causal}: {want:.5f} by the formula, {got:.5f} by differences")
            assert abs(got - want) <= 0.02 * max(abs(want), 0.01), (name, causal, want, got)


def test_token_by_token_is_the_whole_pass(example):
    """fp32: both ways form the same sums in other orders; each is off by less than 2^-24 times the longest chain (70
    keys, 256 products: < 400) times the magnitudes, which are under 20 here; two passes: 1e-3."""
    import torch

    whole, parts = example.generate(dtype=torch.float32)
    assert (whole - parts).abs().max().item() < 1e-3


def test_main_runs(example, capsys):
    example.main(["--steps", "2", "--side", "6"])
    assert "token by token" in capsys.readouterr().out
