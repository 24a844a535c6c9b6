"""Gradients of several micro-batches in the example's layer: every parameter's, the norms' among them, is the sum over the calls."""
import pytest
import torch

from examples import fp8_layer

pytestmark = pytest.mark.gpu

NAMES = ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "norm1", "norm2")


def gradients(layer):
    return {n: (getattr(layer, "d" + n) if n.startswith("norm") else getattr(layer, n).grad).clone() for n in NAMES}


def test_gradients_of_micro_batches_add_up():
    T, C, Hq, Hkv, D, F = 130, 256, 2, 1, 128, 520
    torch.manual_seed(3)
    cos, sin = fp8_layer.rope_tables(T, D, "cuda")
    batches = [[torch.randn(T, C, device="cuda").to(torch.bfloat16) for _ in range(4)] for _ in range(3)]
    new = lambda: fp8_layer.Layer(C, Hq, Hkv, D, F, seed=11)  # noqa: E731

    def step(layer, x, res, dy, dstream):
        layer.backward(dy, dstream, layer.forward(x, res, cos, sin)[2], cos, sin)
        return gradients(layer)

    alone = [step(new(), *b) for b in batches]
    layer = new()
    got = [step(layer, *b) for b in batches][-1]
    for n in NAMES:
        assert got[n].dtype == torch.float32, n
        # each call's term is what it is alone; fp32 additions in the order of the calls
        assert torch.equal(got[n], (alone[0][n] + alone[1][n]) + alone[2][n]), n
        assert not torch.equal(got[n], alone[2][n]), n
