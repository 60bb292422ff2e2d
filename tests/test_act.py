"""Activations stored in 8 bits: codes and steps bit for bit against the definition, what decoding gives,
unbiasedness, values that are not finite, and refusals."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import act_reference as ref
from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)     # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    return zipml.lib()


def values(rows, cols, seed, kind):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(2.0 * rng.standard_normal((1, cols)))
    t = torch.from_numpy(x.astype(np.float32))
    return t if kind == "f32" else t.to(torch.bfloat16)


def stored(x, ld, seed, epoch, tag):
    """(codes, bytes, decoded) of host values x through the library, rows ld apart, everything around them NaN."""
    rows, cols = x.shape
    wide = torch.full((rows, ld), float("nan"), dtype=x.dtype)
    wide[:, :cols] = x
    n = zipml.act_bytes(rows, cols)
    act = torch.full((n + 64,), 0xAB, dtype=torch.uint8, device=DEV)
    zipml.act_encode(wide.to(DEV), rows, cols, ld, seed, epoch, tag, act)
    out = torch.full((rows, ld + 3), 7.0, dtype=x.dtype, device=DEV)
    zipml.act_decode(act, rows, cols, out, ld + 3)
    out, raw = out.cpu().float().numpy(), act.cpu().numpy()
    assert (raw[n:] == 0xAB).all() and (out[:, cols:] == 7.0).all()      # nothing beside its own place
    pitch = -(-cols // 32) * 32
    return raw[:rows * pitch].view(np.int8).reshape(rows, pitch), raw[rows * pitch:n].reshape(rows, pitch // 32), out[:, :cols]


def same(x, ld, seed, epoch, tag):
    codes, byte, out = stored(x, ld, seed, epoch, tag)
    c, b = ref.encode(x.float().numpy(), seed, epoch, tag)
    np.testing.assert_array_equal(byte, b)
    np.testing.assert_array_equal(codes, c)
    np.testing.assert_array_equal(out, ref.decode(c, b, x.shape[1]).astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 2048, 0), (3, 31, 1), (5, 32, 0), (7, 33, 2), (2, 64, 8),
                                           (130, 70, 5), (64, 1021, 3), (1000, 8, 0), (9, 2056, 8), (33, 4104, 0)])
def test_codes_steps_and_values(kind, rows, cols, pad):
    x = values(rows, cols, rows * 7 + cols, kind)
    same(x, cols + pad, 0x1234567890ABCDEF, 77, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_steps_at_their_thresholds(kind):
    """Largest values on both sides of 127 * 2^e, the least and the largest exponents, zeros, subnormal values."""
    tops = [127.0, 128.0, 126.0, 127.5, 1.0, 2.0 ** -126, 2.0 ** -119 * 127 / 128, 2.0 ** -130, 2.0 ** -133, 0.0, 3.3e38,
            2.0 ** 127, -127.0, -128.0, 2.0 ** -120]
    x = torch.zeros(len(tops), 40, dtype=torch.float32)
    x[:, 5] = torch.tensor(tops)
    x[:, 9] = torch.tensor(tops) * 0.37
    x[:, 33] = -torch.tensor(tops)
    x = x if kind == "f32" else x.to(torch.bfloat16)
    same(x, 40, 5, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_groups_that_are_not_finite_decode_to_nan(kind):
    x = values(6, 96, 1, kind)
    x[0, 3], x[1, 40], x[2, 95], x[3, 64] = float("nan"), float("inf"), float("-inf"), float("nan")
    _, byte, out = stored(x, 96, 9, 1, 2)
    where = {0: 0, 1: 1, 2: 2, 3: 2}
    for r in range(6):
        for g in range(3):
            group = out[r, 32 * g:32 * g + 32]
            if where.get(r) == g:
                assert byte[r, g] == 255 and np.isnan(group).all()
            else:
                assert byte[r, g] != 255 and np.isfinite(group).all()
    same(x, 99, 9, 1, 2)


@pytest.mark.gpu
def test_decoding_to_the_other_type():
    x = values(17, 50, 4, "f32")
    act = torch.zeros(zipml.act_bytes(17, 50), dtype=torch.uint8, device=DEV)
    zipml.act_encode(x.to(DEV), 17, 50, 50, 1, 2, 3, act)
    a = torch.zeros(17, 50, dtype=torch.float32, device=DEV)
    b = torch.zeros(17, 50, dtype=torch.bfloat16, device=DEV)
    zipml.act_decode(act, 17, 50, a, 50)
    zipml.act_decode(act, 17, 50, b, 50)
    assert torch.equal(a, b.float())                   # every value is a bf16 number


@pytest.mark.gpu
def test_unbiased_over_seeds():
    """The mean over n independent draws is within 6 standard errors: a step's rounding has variance at most
    step^2 / 4, so 6 * step / (2 sqrt(n)); 2^-17 of a step is the definition's own."""
    x = values(4, 64, 2, "f32")
    n = 2000
    act = torch.zeros(zipml.act_bytes(4, 64), dtype=torch.uint8, device=DEV)
    out = torch.zeros(4, 64, dtype=torch.float32, device=DEV)
    total = torch.zeros(4, 64, dtype=torch.float64, device=DEV)
    xd = x.to(DEV)
    for s in range(n):
        zipml.act_encode(xd, 4, 64, 64, s, 0, 0, act)
        zipml.act_decode(act, 4, 64, out, 64)
        total += out
    step = np.repeat(np.exp2(ref.encode(x.numpy())[1] - 127.0), 32, axis=1)
    off = np.abs((total / n).cpu().numpy() - x.double().numpy())
    assert (off <= step * (3.0 / np.sqrt(n) + 2.0 ** -17)).all()


@pytest.mark.gpu
def test_on_another_stream():
    """The work goes to the stream that is given, behind what that stream already holds."""
    side = torch.cuda.Stream()
    x = values(512, 512, 8, "bf16")
    act = torch.zeros(zipml.act_bytes(512, 512), dtype=torch.uint8, device=DEV)
    xd = torch.zeros(512, 512, dtype=torch.bfloat16, device=DEV)
    host = x.pin_memory()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        xd.copy_(host, non_blocking=True)
    zipml.act_encode(xd, 512, 512, 512, 3, 0, 0, act, stream=side)
    side.synchronize()
    c, b = ref.encode(x.float().numpy(), 3, 0, 0)
    np.testing.assert_array_equal(act.cpu().numpy(), ref.pack(c, b))


@pytest.mark.gpu
def test_the_current_stream_is_the_default():
    side = torch.cuda.Stream()
    assert zipml._stream() == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert zipml._stream() == side.cuda_stream
    assert zipml._stream(side) == side.cuda_stream


def test_sizes(lib):
    assert zipml.act_bytes(1, 1) == 33
    assert zipml.act_bytes(10, 64) == 660
    assert zipml.act_bytes(1000, 70) == 1000 * 99
    for rows, cols in ((0, 5), (5, 0), (-1, 5), (1 << 41, 1), (1, 1 << 31), (1 << 40, 1 << 20)):
        assert zipml.act_bytes(rows, cols) == 0


def test_refusals(lib):
    def enc(x=FAKE, dtype=zipml.BF16, rows=4, cols=40, ld=40, epoch=0, tag=0, act=FAKE):
        return lib.zipml_act_encode(None, x, dtype, rows, cols, ld, 0, epoch, tag, act)
    for kw in ({"x": None}, {"act": None}, {"rows": 0}, {"cols": 0}, {"rows": -3}, {"ld": 39}, {"dtype": 2},
               {"dtype": -1}, {"epoch": 1 << 24}, {"tag": -1}, {"tag": 240}, {"ld": 1 << 60}, {"cols": 1 << 31, "ld": 1 << 31}):
        assert enc(**kw) == zipml.EINVAL, kw
    assert enc(x=ODD) == zipml.EALIGN and enc(act=ODD) == zipml.EALIGN

    def dec(act=FAKE, rows=4, cols=40, out=FAKE, dtype=zipml.F32, ld=40):
        return lib.zipml_act_decode(None, act, rows, cols, out, dtype, ld)
    for kw in ({"act": None}, {"out": None}, {"rows": 0}, {"cols": -1}, {"ld": 39}, {"dtype": 7}):
        assert dec(**kw) == zipml.EINVAL, kw
    assert dec(out=ODD) == zipml.EALIGN and dec(act=ODD) == zipml.EALIGN


def test_types_the_library_does_not_have_are_refused(lib):
    assert zipml._dtype(torch.float16) == -1 and zipml._dtype(torch.bfloat16) == zipml.BF16
