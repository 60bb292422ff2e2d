"""Tensors whose offsets pass 32 bits, and calls on two streams at once."""
import numpy as np
import pytest
import torch

import act_reference as act
from paper_1611_05402_amd import zipml

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda", torch.bfloat16
ROWS, WIDE = 70000, 40000                                  # 2.8e9 values


@pytest.fixture(scope="module")
def wide():
    return torch.zeros(ROWS, WIDE, dtype=BF16, device=DEV)


def put(wide, cols, seed):
    """Random values in the first `cols` columns of the wide rows, and the same packed."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    wide[:, :cols] = torch.randn(ROWS, cols, generator=g, device=DEV).to(BF16)
    return wide[:, :cols].contiguous()


def test_storing_and_restoring(wide):
    n = zipml.act_bytes(ROWS, WIDE)
    assert n > 1 << 31
    wide.zero_()
    rng = np.random.default_rng(1)
    tail = torch.from_numpy(rng.standard_normal((2, WIDE)).astype(np.float32)).to(BF16)
    wide[-2:] = tail.to(DEV)
    stored = torch.empty(n, dtype=torch.uint8, device=DEV)
    zipml.act_encode(wide, ROWS, WIDE, WIDE, 3, 4, 5, stored)
    c, b = act.encode(tail.float().numpy(), 3, 4, 5, row0=ROWS - 2)
    assert np.array_equal(stored[(ROWS - 2) * WIDE:ROWS * WIDE].view(torch.int8).cpu().numpy(), c.reshape(-1))
    assert np.array_equal(stored[-2 * (WIDE // 32):].cpu().numpy(), b.reshape(-1))
    wide.fill_(7.0)
    zipml.act_decode(stored, ROWS, WIDE, wide, WIDE)
    assert np.array_equal(wide[-2:].float().cpu().numpy(), act.decode(c, b, WIDE).astype(np.float32))
    assert (wide[:-2:997] == 0).all()


def test_weight_gradient(wide):
    dy = put(wide, 24, 2)
    x = torch.randn(ROWS, 32, device=DEV).to(BF16)
    stored = torch.empty(zipml.act_bytes(ROWS, 32), dtype=torch.uint8, device=DEV)
    zipml.act_encode(x, ROWS, 32, 32, 1, 0, 0, stored)
    ws = torch.empty(zipml.act_wgrad_workspace_bytes(ROWS, 24, 32, BF16), dtype=torch.uint8, device=DEV)
    out = [torch.zeros(24, 32, device=DEV) for _ in range(2)]
    zipml.act_wgrad(dy, 24, stored, ROWS, 24, 32, out[0], 32, ws)
    zipml.act_wgrad(wide, WIDE, stored, ROWS, 24, 32, out[1], 32, ws)
    assert out[0].abs().sum() > 0 and torch.equal(*out)


def test_recurrence(wide):
    """x, z, dy and the outputs as columns of the wide rows against the same packed."""
    c = 40
    xz, dy = put(wide, 2 * c, 3), torch.randn(ROWS, c, device=DEV).to(BF16)
    start = torch.tensor([0, 5, ROWS - 300, ROWS], device=DEV)
    ws = torch.empty(zipml.scan_workspace_bytes(ROWS, c), dtype=torch.uint8, device=DEV)
    got = []
    for src, ld, y in ((xz, 2 * c, torch.zeros(ROWS, c, dtype=BF16, device=DEV)), (wide, WIDE, wide[:, 1000:])):
        ax, az = (torch.empty(zipml.act_bytes(ROWS, c), dtype=torch.uint8, device=DEV) for _ in range(2))
        states = torch.empty(-(-ROWS // zipml.SCAN_BLOCK), c, device=DEV)
        zipml.scan_forward(src, ld, src[:, c:], ld, ROWS, c, y, y.stride(0), ws, seq_start=start, n_seq=3, act_x=ax, act_z=az,
                           states=states, seed=9)
        g = wide[:, 2000:] if src is wide else torch.zeros(ROWS, 2 * c, dtype=BF16, device=DEV)
        zipml.scan_backward(ax, az, states, dy, c, ROWS, c, g, g.stride(0), g[:, c:], g.stride(0), ws, seq_start=start, n_seq=3)
        got.append((y[:, :c].contiguous(), g[:, :2 * c].contiguous(), ax, az))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Chains of two calls side by side on one card: each waits only for its own, and the results are those of one alone."""
    t, c = 30000, 256
    streams = [torch.cuda.Stream() for _ in range(2)]
    x = [torch.randn(t, 2 * c, device=DEV).to(BF16) for _ in range(2)]
    ws = [torch.empty(zipml.scan_workspace_bytes(t, c), dtype=torch.uint8, device=DEV) for _ in range(2)]
    alone = []
    for k in range(2):
        y = torch.empty(t, c, dtype=BF16, device=DEV)
        zipml.scan_forward(x[k], 2 * c, x[k][:, c:], 2 * c, t, c, y, c, ws[k])
        alone.append(y)
    torch.cuda.synchronize()
    both = [[torch.empty(t, c, dtype=BF16, device=DEV) for _ in range(6)] for _ in range(2)]
    for n in range(6):
        for k in range(2):
            zipml.scan_forward(x[k], 2 * c, x[k][:, c:], 2 * c, t, c, both[k][n], c, ws[k], stream=streams[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(alone[k], y) for y in both[k])


def test_large_results_are_those_of_small_ones():
    """More than 96 MiB are written another way; the values are the same, and the rows' padding stays as it was."""
    rows, cols = 6200, 4099
    x = torch.randn(rows, cols, device=DEV)
    stored = torch.empty(zipml.act_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    zipml.act_encode(x, rows, cols, cols, 1, 2, 3, stored)
    small = torch.full((rows, cols + 3), 9.0, dtype=BF16, device=DEV)
    large = torch.full((rows, cols + 3), 9.0, device=DEV)
    assert rows * cols * 2 < 96 << 20 < rows * cols * 4
    zipml.act_decode(stored, rows, cols, small, cols + 3)
    zipml.act_decode(stored, rows, cols, large, cols + 3)
    assert torch.equal(small.float(), large) and (large[:, cols:] == 9.0).all()
