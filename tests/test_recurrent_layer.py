"""The layer of examples/recurrent_layer.py: it learns, its gradients are those of the layer, and it serves."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_layer.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("recurrent_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_learns_and_serves(ex):
    losses, layer = ex.train(steps=40, tokens=1000, d_in=64, channels=96, d_out=40, n_seq=5, say=lambda *a: None)
    assert np.isfinite(losses).all() and np.mean(losses[-5:]) < 0.5 * np.mean(losses[:5])
    # both ways round y to bf16 once and multiply it by the same weights: a few units of 2^-8
    assert ex.serve(layer, say=lambda *a: None) < 0.03


def test_gradients_are_those_of_the_layer(ex):
    """Against automatic differentiation in fp32 of the same layer without stored activations.  A stored value is off by
    less than a step, at most 2/127 of its group's largest, in random directions: over 600 tokens the relative error of a
    weight gradient's norm stays below 5 %."""
    tokens, d, c, o, n = 600, 64, 64, 32, 4
    layer = ex.RecurrentLayer(d, c, o, tokens, n, seed=4)
    g = torch.Generator(device=ex.DEV)
    g.manual_seed(5)
    u = torch.randn(tokens, d, generator=g, device=ex.DEV).to(ex.BF16)
    d_out = torch.randn(tokens, o, generator=g, device=ex.DEV).to(ex.BF16)
    start = ex.documents(tokens, n, 6)
    layer.forward(u, start)
    du = layer.backward(d_out, start)

    w_in, w_out = (w.float().cpu().requires_grad_() for w in (layer.b_in, layer.b_out))
    uf = u.float().cpu().requires_grad_()
    xz = uf @ w_in.t()
    ys, h = [], None
    first = set(start.cpu().tolist()[:-1])
    for t in range(tokens):
        f = torch.sigmoid(xz[t, c:])
        prev = torch.zeros(c) if t in first or h is None else h
        h = f * prev + (1 - f) * xz[t, :c]
        ys.append(h)
    (torch.stack(ys) @ w_out.t() * d_out.float().cpu()).sum().backward()
    for got, want in ((layer.dw_in, w_in.grad), (layer.dw_out, w_out.grad), (du.float(), uf.grad)):
        off = (got.cpu() - want).norm() / want.norm()
        assert off < 0.05, float(off)
