"""A wait of the recurrence's blocks that gives up (forced from the host: no polls allowed) is reported, and the next call is right again."""
import ctypes as C
import os

import pytest
import torch

from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)


def test_refusals():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    status = zipml.lib().zipml_scan_status
    assert status(None, None, 1 << 20) == zipml.EWORKSPACE and status(None, FAKE, 8) == zipml.EWORKSPACE
    assert status(None, ODD, 1 << 20) == zipml.EALIGN


def scan(tokens, c, ws):
    g = torch.Generator(device=DEV)
    g.manual_seed(tokens)
    xz = torch.randn(tokens, 2 * c, generator=g, device=DEV)
    y = torch.empty(tokens, c, device=DEV)
    kept = dict(act_x=torch.empty(zipml.act_bytes(tokens, c), dtype=torch.uint8, device=DEV),
                act_z=torch.empty(zipml.act_bytes(tokens, c), dtype=torch.uint8, device=DEV),
                states=torch.empty(-(-tokens // zipml.SCAN_BLOCK), c, device=DEV))
    zipml.scan_forward(xz, 2 * c, xz[:, c:], 2 * c, tokens, c, y, c, ws, **kept)
    first = zipml.scan_status(ws)
    dx, dz = torch.empty(tokens, c, device=DEV), torch.empty(tokens, c, device=DEV)
    zipml.scan_backward(kept["act_x"], kept["act_z"], kept["states"], y, c, tokens, c, dx, c, dz, c, ws)
    return (first, bool(torch.isnan(y).any())), (zipml.scan_status(ws), bool(torch.isnan(dx).any()), bool(torch.isnan(dz).any()))


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,c", [(16384, 128), (65536, 1024)])      # 256 workgroups of 32 channels, 4,096 of 64
def test_a_wait_that_gives_up_is_reported(tokens, c, knobs):
    """Hundreds of blocks that start together cannot all find the state of the one before them at their first look."""
    ws = torch.full((zipml.scan_workspace_bytes(tokens, c),), 0xFF, dtype=torch.uint8, device=DEV)
    right = (zipml.OK, False), (zipml.OK, False, False)
    assert scan(tokens, c, ws) == right
    knobs(zipml.KNOB_SPIN_LIMIT, 0)
    (status, nan), (back, _, _) = scan(tokens, c, ws)
    assert status == zipml.ETIMEOUT and nan and back == zipml.ETIMEOUT
    knobs(zipml.KNOB_SPIN_LIMIT, -1)
    assert scan(tokens, c, ws) == right


@pytest.mark.gpu
def test_a_single_block_waits_for_nothing(knobs):
    ws = torch.full((zipml.scan_workspace_bytes(200, 72),), 0xFF, dtype=torch.uint8, device=DEV)
    knobs(zipml.KNOB_SPIN_LIMIT, 0)
    assert scan(200, 72, ws) == ((zipml.OK, False), (zipml.OK, False, False))
