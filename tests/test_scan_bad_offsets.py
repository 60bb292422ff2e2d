"""Offsets that do not ascend or lie outside the tokens: what the calls give is undefined, but nothing outside the arrays is written.  Every array that
a call writes lies between guards of 4 KiB, rows lie apart with guards between them."""
import numpy as np
import pytest
import torch

from paper_1611_05402_amd import zipml

pytestmark = pytest.mark.gpu
DEV, GUARD, MARK = "cuda", 4096, 0xA5


class Guarded:
    def __init__(self):
        self.raw = []

    def array(self, *shape, dtype=torch.float32):
        n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
        buf = torch.full((GUARD + -(-n // 16) * 16 + GUARD,), MARK, dtype=torch.uint8, device=DEV)
        self.raw.append((buf, n))
        return buf[GUARD:GUARD + n].view(dtype).view(*shape)

    def check(self):
        for buf, n in self.raw:
            assert (buf[:GUARD] == MARK).all() and (buf[GUARD + n:] == MARK).all()


def offsets(name, tokens):
    rng = np.random.default_rng(7)
    return {"back and forth": [0, 500, 100, 400, 300, tokens],
            "outside": [-70, 20, 9000, 1 << 20],
            "descending": [tokens, 0],
            "far outside": [1 << 40, -(1 << 40), 7, -(1 << 62), 1 << 62],
            "all negative": [-5, -3, -1],
            "many": rng.integers(-300, tokens + 300, 5001),        # more than a block looks through: it searches
            "many descending": np.arange(tokens + 3000, tokens - 3000, -1),
            "many the same": np.full(4000, tokens // 2)}[name]


NAMES = ["back and forth", "outside", "descending", "far outside", "all negative", "many", "many descending", "many the same"]


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,c", [(600, 24), (2500, 1000)])     # workgroups of 32 channels and of 64
@pytest.mark.parametrize("name", NAMES)
def test_nothing_else_is_written(name, tokens, c, kind):
    start = torch.tensor(np.asarray(offsets(name, tokens), np.int64), device=DEV)
    n, pad, a = start.numel() - 1, 16, Guarded()
    x, z, dy = (torch.randn(tokens, c, device=DEV).to(kind) for _ in range(3))
    h0, dh_last = torch.randn(n, c, device=DEV), torch.randn(n, c, device=DEV)
    y, dx, dz = (a.array(tokens, c + pad, dtype=kind) for _ in range(3))
    h_last, dh0, states = a.array(n, c), a.array(n, c), a.array(-(-tokens // zipml.SCAN_BLOCK), c)
    ax, az = (a.array(zipml.act_bytes(tokens, c), dtype=torch.uint8) for _ in range(2))
    ws = a.array(zipml.scan_workspace_bytes(tokens, c), dtype=torch.uint8)
    zipml.scan_forward(x, c, z, c, tokens, c, y, c + pad, ws, seq_start=start, n_seq=n, h0=h0, h_last=h_last, act_x=ax, act_z=az,
                       states=states)
    assert zipml.scan_status(ws) == zipml.OK
    zipml.scan_backward(ax, az, states, dy, c, tokens, c, dx, c + pad, dz, c + pad, ws, seq_start=start, n_seq=n, h0=h0,
                        dh_last=dh_last, dh0=dh0)
    assert zipml.scan_status(ws) == zipml.OK
    a.check()
    for t in (y, dx, dz):
        assert (t.view(torch.uint8).view(tokens, -1)[:, c * t.element_size():] == MARK).all()
