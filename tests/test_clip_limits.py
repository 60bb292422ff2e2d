"""Clipping with an infinite largest norm, which scales nothing: gradients that are finite, that hold an infinity, that hold a NaN."""
import math

import pytest
import torch

from paper_1611_05402_amd import zipml

DEV, INF = "cuda", float("inf")
SIZES = [700, 3, 20001]


def run(bad=None):
    g = torch.Generator(device=DEV).manual_seed(1)
    grads = [torch.randn(n, generator=g, device=DEV) for n in SIZES]
    if bad is not None:
        grads[1][2] = bad
    before, outs = [t.clone() for t in grads], [torch.empty_like(t, dtype=torch.bfloat16) for t in grads]
    norm, ws = torch.empty(2, device=DEV), torch.empty(zipml.clip_workspace_bytes(len(SIZES)), dtype=torch.uint8, device=DEV)
    zipml.clip(zipml.ClipList(grads, outs), INF, norm, ws)
    zipml.clip(zipml.ClipList(grads), INF, norm, ws)
    return before, grads, outs, norm.tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [None, INF, -INF])
def test_an_infinite_largest_norm_scales_nothing(bad):
    before, grads, outs, (norm, factor) = run(bad)
    want = math.sqrt(sum(float(t.double().square().sum()) for t in before))
    # one rounding to fp32, and a 64-bit sum in another order
    assert factor == 1.0 and (norm == want if bad else abs(norm - want) <= 2.0 ** -24 * want * (1 + 1e-6))
    for b, t, o in zip(before, grads, outs):
        assert torch.equal(t, b) and torch.equal(o, b.to(torch.bfloat16))


@pytest.mark.gpu
def test_a_nan_shows_with_an_infinite_largest_norm():
    _, grads, outs, (norm, factor) = run(float("nan"))
    assert math.isnan(norm) and math.isnan(factor) and all(torch.isnan(t).all() for t in grads + outs)
