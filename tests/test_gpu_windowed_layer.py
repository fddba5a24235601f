"""The operators over pages and packed rows together, as examples/windowed_layer.py runs them: what a layer serves token by token is what
it computes over whole sequences, and its gradients are the slopes of its own forward pass."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("windowed_layer", os.path.join(ROOT, "examples", "windowed_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("S, lo, hi, steps, page", [(24, 5, 900, 40, 16), (3, 1, 3, 30, 8), (1, 700, 700, 3, 64)])
def test_serving_and_training_compute_the_same(example, S, lo, hi, steps, page):
    """bf16: each side rounds q, k, v, the probabilities and the outputs once (2^-8 each at most, in all directions), and the output
    projection adds up independent ones."""
    far, _ = example.main(S, lo, hi, steps, page, quiet=True)
    assert far < 2.0 ** -7


def test_the_layers_gradients_are_slopes(example):
    """Along a direction of every parameter the sum of dy times the change of y is what the gradients say.  The change is measured with
    steps large enough that bf16 outputs resolve it: 2^-8 of rounding in y against steps of 2^-3 leaves a few percent over many rows."""
    layer = example.Layer(d=256, n_q=4, n_kv=2, h=64, window=50, sinks=2)
    lens = [70, 1, 130]
    starts = torch.tensor([0, 70, 71, 201], dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n) for n in lens]).int().cuda()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(201, 256, generator=g, device="cuda").bfloat16()
    y, saved = layer.forward(x, starts, pos, 130)
    dy = torch.randn(y.shape, generator=g, device="cuda").bfloat16()
    grads = layer.backward(dy, saved)
    for name in ("q_gain", "k_gain"):
        before = getattr(layer, name)
        # along the gradient itself, so that the slope is as large as it gets
        e = grads[name] / grads[name].norm()
        t = 0.25
        setattr(layer, name, before + t * e)
        up = layer.forward(x, starts, pos, 130)[0]
        setattr(layer, name, before - t * e)
        down = layer.forward(x, starts, pos, 130)[0]
        setattr(layer, name, before)
        slope = float(((up.double() - down.double()) * dy.double()).sum() / (2 * t))
        want = float(grads[name].norm())
        # rounding: two outputs of 2^-9 of their size each (root mean square below 2^-9), against dy, over the step
        noise = 4 * 2.0 ** -9 * float((y.double() * dy.double()).norm()) / t
        assert abs(slope - want) <= 0.05 * want + noise, (name, slope, want, noise)
