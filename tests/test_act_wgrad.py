"""The weight gradient from stored activations against the same sums in 64 bits.

Products are exact and every sum of n terms is taken in fp32 in some order, so an element is within
n * 2^-24 * sum |terms| of the exact one, whatever the order (n + 8 here: joining parts, adding to dW)."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import act_reference as ref
from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    return zipml.lib()


def inputs(rows, d_out, d_in, kind, seed=0):
    rng = np.random.default_rng(seed + rows + 3 * d_out + 7 * d_in)
    dy = torch.from_numpy((rng.standard_normal((rows, d_out)) * 0.02).astype(np.float32))
    x = (rng.standard_normal((rows, d_in)) * np.exp(rng.standard_normal((1, d_in)))).astype(np.float32)
    codes, byte = ref.encode(x, seed)
    return dy if kind == "f32" else dy.to(torch.bfloat16), codes, byte


def wgrad(dy, codes, byte, d_in, pad_y=0, pad_w=0, flags=0, before=None):
    rows, d_out = dy.shape
    wide = torch.full((rows, d_out + pad_y), float("nan"), dtype=dy.dtype)
    wide[:, :d_out] = dy
    dw = torch.full((d_out, d_in + pad_w), 5.0, dtype=torch.float32, device=DEV)
    if before is not None:
        dw[:, :d_in] = torch.from_numpy(before).to(DEV)
    act = torch.from_numpy(ref.pack(codes, byte)).to(DEV)
    ws = torch.full((zipml.act_wgrad_workspace_bytes(rows, d_out, d_in, dy.dtype),), 0xFF, dtype=torch.uint8, device=DEV)
    zipml.act_wgrad(wide.to(DEV), d_out + pad_y, act, rows, d_out, d_in, dw, d_in + pad_w, ws, flags=flags)
    out = dw.cpu().numpy()
    assert (out[:, d_in:] == 5.0).all()
    return out[:, :d_in]


def check(dy, codes, byte, d_in, out, before=None):
    a, b = dy.double().numpy(), ref.decode(codes, byte, d_in)
    want, size = a.T @ b, np.abs(a).T @ np.abs(b)
    if before is not None:
        want, size = want + before, size + np.abs(before)
    assert (np.abs(out - want) <= (dy.shape[0] + 8) * 2.0 ** -24 * size).all()


SIZES = [(1, 1, 1), (1, 300, 70), (2, 16, 33), (31, 129, 31), (64, 128, 128), (65, 127, 257), (200, 40, 300),
         (1000, 130, 129), (3001, 64, 96)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d_out,d_in", SIZES)
def test_against_64_bits(kind, rows, d_out, d_in):
    dy, codes, byte = inputs(rows, d_out, d_in, kind)
    for pad_y in (0, 3, 8):
        check(dy, codes, byte, d_in, wgrad(dy, codes, byte, d_in, pad_y, pad_y // 2))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d_out,d_in", [(150, 2600, 3100), (257, 4099, 2050)])
def test_large_layers(kind, rows, d_out, d_in):
    dy, codes, byte = inputs(rows, d_out, d_in, kind)
    check(dy, codes, byte, d_in, wgrad(dy, codes, byte, d_in, 5))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d_out,d_in", [(2500, 520, 390), (700, 1030, 900), (6000, 260, 700), (20000, 130, 250),
                                             (1990, 2100, 1500), (40000, 500, 256)])
def test_middle_sizes(kind, rows, d_out, d_in):
    """Where tiles of 128 and 256, in one range of tokens and in several, take over from each other."""
    dy, codes, byte = inputs(rows, d_out, d_in, kind)
    check(dy, codes, byte, d_in, wgrad(dy, codes, byte, d_in, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [321, 384, 400, 449, 512, 577, 640, 700, 961])
def test_rounds_of_tokens_shared_by_turns(kind, rows):
    """Numbers of tokens that leave some of a turn's rounds short or empty."""
    dy, codes, byte = inputs(rows, 131, 70, kind)
    for flags, before in ((0, None), (zipml.WGRAD_ADD, np.full((131, 70), 0.25, np.float32))):
        check(dy, codes, byte, 70, wgrad(dy, codes, byte, 70, 1, 1, flags, before), before)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d_out", [5, 130])
def test_rows_far_apart(kind, d_out):
    """Rows of dY more than 16 MiB apart are read value by value."""
    dy, codes, byte = inputs(3, d_out, 70, kind)
    check(dy, codes, byte, 70, wgrad(dy, codes, byte, 70, (1 << 24) // dy.element_size() + 3))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out", [(1, 1), (1, 63), (64, 65), (129, 255), (500, 129), (300, 4097)])
def test_the_very_last_value_of_dy(rows, d_out):
    """An odd number of bf16 values a row: the last value of the last row counts, and nothing behind it is read as one."""
    dy, codes, byte = inputs(rows, d_out, 45, "bf16")
    dy[-1, -1] = 3.0
    codes[-1, :45] = 100
    for pad in (0, 1, 2):
        check(dy, codes, byte, 45, wgrad(dy, codes, byte, 45, pad))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out,d_in", [(2500, 521, 390), (6000, 257, 700), (20000, 131, 250), (5000, 1, 3000)])
def test_the_last_value_of_every_range_of_tokens(rows, d_out, d_in):
    """The same where the tokens are taken in several ranges, which end at multiples of 64 tokens."""
    dy, codes, byte = inputs(rows, d_out, d_in, "bf16")
    dy[:, -1] = 0
    dy[63::64, -1] = 3.0
    for pad in (0, 1, 2):
        check(dy, codes, byte, d_in, wgrad(dy, codes, byte, d_in, pad))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d_out,d_in", [(5, 9, 40), (3000, 100, 65)])
def test_adding_to_what_is_there(kind, rows, d_out, d_in):
    dy, codes, byte = inputs(rows, d_out, d_in, kind)
    before = np.random.default_rng(1).standard_normal((d_out, d_in)).astype(np.float32)
    check(dy, codes, byte, d_in, wgrad(dy, codes, byte, d_in, 0, 1, zipml.WGRAD_ADD, before), before)


@pytest.mark.gpu
def test_fp32_gradients_keep_their_24_bits():
    """One token: dW is a single product, exact up to its one rounding to fp32."""
    dy, codes, byte = inputs(1, 200, 100, "f32", 3)
    want = (dy.double().numpy().T @ ref.decode(codes, byte, 100)).astype(np.float32)
    out = wgrad(dy, codes, byte, 100)
    assert (np.abs(out.astype(np.float64) - want) <= 2.0 ** -22 * np.abs(want)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_values_that_are_not_finite(kind):
    """A NaN group reaches its 32 columns, an infinite or NaN dY its row; the rest stays finite."""
    dy, codes, byte = inputs(40, 50, 96, kind)
    dy[7, 11], dy[9, 13] = float("inf"), float("nan")
    byte[5, 1], codes[5, 32:64] = 255, 0
    codes[7, :32] = 3                                       # infinity times a code other than 0
    out = wgrad(dy, codes, byte, 96)
    assert np.isnan(out[:, 32:64]).all() and np.isnan(out[13]).all() and np.isinf(out[11, :32]).all()
    rest = np.delete(np.delete(out, np.s_[32:64], 1), [11, 13], 0)
    assert np.isfinite(rest).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_large_and_small_dy(kind):
    """dY over the type's range: the terms of an fp32 value neither overflow nor vanish."""
    dy, codes, byte = inputs(64, 96, 40, kind)
    scale = torch.ones(96)
    scale[:32], scale[32:64] = 2.0 ** 100, 2.0 ** -70
    dy = (dy.float() * scale).to(dy.dtype)
    check(dy, codes, byte, 40, wgrad(dy, codes, byte, 40))


@pytest.mark.gpu
def test_same_bits_every_time():
    dy, codes, byte = inputs(5000, 200, 130, "bf16")
    a = wgrad(dy, codes, byte, 130)
    assert all(np.array_equal(a, wgrad(dy, codes, byte, 130)) for _ in range(3))


@pytest.mark.gpu
def test_unbiased_estimate_of_the_exact_gradient():
    """Mean over n draws of Q against dY^T X: within 6 standard errors, a value's variance being at most step^2 / 4."""
    rng = np.random.default_rng(11)
    rows, d_out, d_in, n = 48, 20, 64, 400
    dy = torch.from_numpy(rng.standard_normal((rows, d_out)).astype(np.float32))
    x = rng.standard_normal((rows, d_in)).astype(np.float32)
    xd, dyd = torch.from_numpy(x).to(DEV), dy.to(DEV)
    act = torch.zeros(zipml.act_bytes(rows, d_in), dtype=torch.uint8, device=DEV)
    ws = torch.zeros(zipml.act_wgrad_workspace_bytes(rows, d_out, d_in, torch.float32), dtype=torch.uint8, device=DEV)
    dw = torch.zeros(d_out, d_in, dtype=torch.float32, device=DEV)
    for s in range(n):
        zipml.act_encode(xd, rows, d_in, d_in, s, 0, 0, act)
        zipml.act_wgrad(dyd, d_out, act, rows, d_out, d_in, dw, d_in, ws, flags=zipml.WGRAD_ADD)
    step = np.repeat(np.exp2(ref.encode(x)[1] - 127.0), 32, axis=1)
    spread = np.sqrt((dy.numpy().astype(np.float64) ** 2).T @ (step ** 2 / 4.0) / n)
    off = np.abs(dw.cpu().numpy() / n - dy.numpy().astype(np.float64).T @ x)
    assert (off <= 6.0 * spread + 1e-4).all()


def test_sizes(lib):
    f, b = torch.float32, torch.bfloat16
    assert zipml.act_wgrad_workspace_bytes(1, 1, 1, b) > 0
    assert zipml.act_wgrad_workspace_bytes(65536, 512, 256, b) >= 512 * 256 * 4
    for rows, o, i in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, (1 << 24) + 1, 1), (1, 1, (1 << 24) + 1), (1, 1 << 20, 1 << 20)):
        assert zipml.act_wgrad_workspace_bytes(rows, o, i, f) == 0
    assert zipml.act_wgrad_workspace_bytes(4, 4, 4, torch.float16) == 0


def test_refusals(lib):
    def call(dy=FAKE, dtype=zipml.BF16, ldy=8, act=FAKE, rows=16, o=8, i=40, flags=0, dw=FAKE, ldw=40, ws=FAKE, n=1 << 24):
        return lib.zipml_act_wgrad(None, dy, dtype, ldy, act, rows, o, i, flags, dw, ldw, ws, n)
    for kw in ({"dy": None}, {"act": None}, {"dw": None}, {"dtype": 2}, {"ldy": 7}, {"ldw": 39}, {"rows": 0}, {"o": 0},
               {"i": 0}, {"flags": 2}, {"flags": -1}, {"ldy": 1 << 60}, {"ldw": 1 << 60}, {"o": 1 << 25, "ldy": 1 << 25}):
        assert call(**kw) == zipml.EINVAL, kw
    assert call(ws=None) == zipml.EWORKSPACE and call(n=8) == zipml.EWORKSPACE
    for kw in ({"dy": ODD}, {"act": ODD}, {"dw": ODD}, {"ws": ODD}):
        assert call(**kw) == zipml.EALIGN, kw
