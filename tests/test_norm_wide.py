"""Rows so wide that the gradient of the gain takes more threads than one launch holds."""
import pytest
import torch

from paper_1611_05402_amd import zipml

DEV = "cuda"


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, zipml.NORM_ADD])
def test_gradients_of_more_than_2_to_the_26_columns(flags):
    """dx stands in the place of dy.  Against 64 bits: dgain is a product of a rounded n with dy, two of them added (and what was there): three
    roundings of 2^-24 of the sizes that are added up, two more to be safe.  dx: the mean of a n is a sum of chains of 2^26 / 1,024 + 8 products
    in each thread and 16 + 6 steps over them, off by at most 66,000 * 2^-24 of the mean of |a n|; the rest is 4 roundings, and one to bf16."""
    rows, cols = 2, (1 << 26) + 37
    g = torch.Generator(device=DEV).manual_seed(1)
    r, dy = ((torch.randn(rows, cols, generator=g, device=DEV) * s).to(torch.bfloat16) for s in (1.0, 0.02))
    rstd = torch.tensor([0.9, 1.2], device=DEV)
    dx = dy.clone()
    start = torch.arange(cols, device=DEV, dtype=torch.float32) % 7 if flags else torch.full((cols,), float("nan"), device=DEV)
    dgain = torch.cat([start, torch.full((3,), 7.0, device=DEV)])
    ws = torch.full((zipml.norm_backward_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device=DEV)
    zipml.norm_backward(dx, cols, r, cols, rows, cols, rstd, dx, cols, ws, dgain=dgain[:cols], flags=flags)
    n, a = r.double() * rstd.double()[:, None], dy.double()
    want, size = (a * n).sum(0), (a * n).abs().sum(0)
    if flags:
        want, size = want + start.double(), size + start.double()
    assert ((dgain[:cols].double() - want).abs() <= 5 * 2.0 ** -24 * size).all() and (dgain[cols:] == 7.0).all()
    along, most = (a * n).mean(1, keepdim=True), (a * n).abs().mean(1, keepdim=True)
    want = rstd.double()[:, None] * (a - n * along)
    off = rstd.double()[:, None] * 2.0 ** -24 * (4 * a.abs() + n.abs() * 66000 * most)
    assert ((dx.double() - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all()


@pytest.mark.gpu
def test_gradients_of_columns_on_both_sides_of_a_launch():
    """A chain of three rows: a rounding of n and one of each sum, 2^-24 of the sizes that are added up."""
    rows, cols = 3, (1 << 25) + 24
    g = torch.Generator(device=DEV).manual_seed(2)
    r, dy = ((torch.randn(rows, cols, generator=g, device=DEV) * s).to(torch.bfloat16) for s in (1.0, 0.02))
    rstd, dgain = torch.tensor([0.9, 1.2, 1.0], device=DEV), torch.full((cols + 1,), 7.0, device=DEV)
    ws = torch.full((zipml.norm_backward_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device=DEV)
    zipml.norm_backward(dy, cols, r, cols, rows, cols, rstd, torch.empty_like(dy), cols, ws, dgain=dgain[:cols])
    each = dy.double() * r.double() * rstd.double()[:, None]
    assert ((dgain[:cols].double() - each.sum(0)).abs() <= 6 * 2.0 ** -24 * each.abs().sum(0)).all() and dgain[cols] == 7.0
