"""Linear layer on 8-bit codes, bit for bit: the sums are exact and what follows are single fp32 operations."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import row8_reference as ref
from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD, HALF = C.c_void_p(0x1000), C.c_void_p(0x1004), C.c_void_p(0x1002)     # never dereferenced: the checks come first
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    return zipml.lib()


def codes(rows, cols, seed):
    rng = np.random.default_rng(seed)
    return rng.integers(-127, 128, (rows, cols), dtype=np.int8), (np.exp(rng.standard_normal(rows)) * 0.01).astype(np.float32)


def on_gpu(q, more=0):
    """Rows of codes on the GPU, `more` bytes further apart than they need with 99 in them, zeros in the padding."""
    rows, cols = q.shape
    t = torch.full((rows, ref.pitch(cols) + more), 99, dtype=torch.int8)
    t[:, cols:ref.pitch(cols)] = 0
    t[:, :cols] = torch.from_numpy(q)
    return t.to(DEV)


def product(x, w, sx, sw, bias, kind, more=0, pad=0):
    rows, d_in, d_out = x.shape[0], x.shape[1], w.shape[0]
    xd, wd = on_gpu(x, more), on_gpu(w, more)
    y = torch.full((rows + 1, d_out + pad), 7.0, dtype=TYPES[kind], device=DEV)
    ws = torch.full((zipml.row8_product_workspace_bytes(rows, d_out, d_in),), 0xFF, dtype=torch.uint8, device=DEV)
    zipml.row8_product(xd, xd.stride(0), torch.from_numpy(sx).to(DEV), wd, wd.stride(0), torch.from_numpy(sw).to(DEV), rows, d_out, d_in, y,
                       y.stride(0), ws, bias=None if bias is None else torch.from_numpy(bias).to(DEV))
    assert (y[rows:] == 7.0).all() and (y[:, d_out:] == 7.0).all()
    return y[:rows, :d_out].cpu()


def same(rows, d_out, d_in, kind, bias=False, more=0, pad=0):
    (x, sx), (w, sw) = codes(rows, d_in, 1), codes(d_out, d_in, 2)
    b = np.random.default_rng(3).standard_normal(d_out).astype(np.float32) if bias else None
    got, want = product(x, w, sx, sw, b, kind, more, pad), ref.product(x, w, sx, sw, b, TYPES[kind])
    np.testing.assert_array_equal(got.float().numpy(), want.float().numpy())


SIZES = [(r, o, i) for r in (1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 64, 65, 130) for o, i in ((1, 1), (17, 16), (130, 129), (257, 1001), (520, 2048))]
SIZES += [(1, 4096, 4096), (4, 1000, 16000), (64, 1024, 8192), (16, 64, 30000), (48, 33, 65000), (1000, 1001, 520), (257, 255, 4097), (300, 16, 8192),
          (2048, 1024, 256), (1, 1, 131071), (129, 65, 131071), (3000, 300, 17), (700, 2500, 640), (4100, 5, 100), (520, 1300, 9000)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d_out,d_in", SIZES)
def test_bits(kind, rows, d_out, d_in):
    same(rows, d_out, d_in, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 6, 20, 50, 100, 400, 1500])
@pytest.mark.parametrize("d_out,d_in,more,pad", [(1, 33, 16, 3), (100, 500, 48, 0), (1003, 777, 16, 5), (260, 3000, 112, 1)])
def test_bias_strides_and_odd_rows(kind, rows, d_out, d_in, more, pad):
    same(rows, d_out, d_in, kind, True, more, pad)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 16, 40, 200])
def test_largest_sums(rows):
    """Codes of -128 throughout: 2^14 * 131,071 is the largest sum that 32 bits hold."""
    x, w = np.full((rows, 131071), -128, np.int8), np.full((70, 131071), -128, np.int8)
    w[1], w[2, ::2] = 127, 127
    one, got = np.ones(rows, np.float32), None
    got = product(x, w, one, np.ones(70, np.float32), None, "f32")
    np.testing.assert_array_equal(got.numpy(), ref.product(x, w, one, np.ones(70, np.float32), None, torch.float32).numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out,d_in", [(3, 70, 200), (40, 33, 5000), (300, 200, 520)])
def test_scales_of_nan_and_zero(rows, d_out, d_in):
    (x, sx), (w, sw) = codes(rows, d_in, 1), codes(d_out, d_in, 2)
    sx[1], sw[5], sx[2] = np.nan, np.nan, 0.0
    x[1], w[5] = 0, 0
    got = product(x, w, sx, sw, None, "f32")
    assert torch.isnan(got[1]).all() and torch.isnan(got[:, 5]).all()
    assert torch.isnan(got).sum() == rows + d_out - 1
    np.testing.assert_array_equal(got.numpy(), ref.product(x, w, sx, sw, None, torch.float32).numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out", [(600, 40), (40, 600), (5, 3000)])
def test_rows_far_apart(rows, d_out):
    """Rows 4 MiB apart, so that offsets pass 32 bits in one operand or the other; y past 32 bits as well."""
    (x, sx), (w, sw) = codes(rows, 200, 1), codes(d_out, 200, 2)
    ld, ldy = 1 << 22, (1 << 33) // rows

    def far(q):
        t = torch.empty((q.shape[0] - 1) * ld + 208, dtype=torch.int8, device=DEV)
        rows_of = torch.as_strided(t, (q.shape[0], 208), (ld, 1))
        rows_of.copy_(on_gpu(q))
        return t
    xd, wd = far(x), far(w)
    y = torch.empty((rows - 1) * ldy + d_out, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(zipml.row8_product_workspace_bytes(rows, d_out, 200), dtype=torch.uint8, device=DEV)
    zipml.row8_product(xd, ld, torch.from_numpy(sx).to(DEV), wd, ld, torch.from_numpy(sw).to(DEV), rows, d_out, 200, y, ldy, ws)
    got = torch.as_strided(y, (rows, d_out), (ldy, 1)).cpu()
    assert torch.equal(got, ref.product(x, w, sx, sw, None, torch.bfloat16))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out", [(3, 9), (700, 520), (2000, 2049)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_part_of_the_rows(rows, d_out, kind):
    """Codes and scales from any row on (scales and bias are aligned to their type only)."""
    (x, sx), (w, sw) = codes(rows + 17, 300, 1), codes(d_out + 41, 300, 2)
    b = np.random.default_rng(3).standard_normal(d_out + 3).astype(np.float32)
    xd, wd, sxd, swd, bd = on_gpu(x), on_gpu(w), *(torch.from_numpy(v).to(DEV) for v in (sx, sw, b))
    y = torch.empty(rows, d_out, dtype=TYPES[kind], device=DEV)
    ws = torch.empty(zipml.row8_product_workspace_bytes(rows, d_out, 300), dtype=torch.uint8, device=DEV)
    zipml.row8_product(xd[17:], 304, sxd[17:], wd[41:], 304, swd[41:], rows, d_out, 300, y, d_out, ws, bias=bd[3:])
    assert torch.equal(y.cpu(), ref.product(x[17:], w[41:], sx[17:], sw[41:], b[3:], TYPES[kind]))


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out,d_in,kind", [(8300, 6107, 40, "bf16"), (5000, 5121, 130, "f32"), (4096, 12290, 16, "bf16")])
def test_results_larger_than_the_caches(rows, d_out, d_in, kind):
    same(rows, d_out, d_in, kind, True)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,d_out,d_in", [(4400, 4100, 520), (4864, 3841, 1111), (4097, 8192, 128)])
def test_more_tiles_than_compute_units(rows, d_out, d_in, kind):
    """Tiles of several rounds that follow one another in a workgroup, the last of them partly outside."""
    same(rows, d_out, d_in, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out,d_in", [(1, 520, 4096), (30, 64, 30000), (500, 700, 300)])
def test_two_streams_at_once_and_a_graph(rows, d_out, d_in):
    """Each stream with its own workspace; a captured call replayed over other inputs, with eager work between the replays."""
    (x, sx), (w, sw) = codes(rows, d_in, 1), codes(d_out, d_in, 2)
    want = ref.product(x, w, sx, sw, None, torch.float32)
    xd, wd, sxd, swd = on_gpu(x), on_gpu(w), torch.from_numpy(sx).to(DEV), torch.from_numpy(sw).to(DEV)
    need = zipml.row8_product_workspace_bytes(rows, d_out, d_in)

    def call(y, ws, stream=None):
        zipml.row8_product(xd, xd.stride(0), sxd, wd, wd.stride(0), swd, rows, d_out, d_in, y, d_out, ws, stream=stream)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [(torch.empty(rows, d_out, device=DEV), torch.empty(need, dtype=torch.uint8, device=DEV)) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (y, ws) in zip(streams, outs):
            call(y, ws, s)
    torch.cuda.synchronize()
    for y, _ in outs:
        np.testing.assert_array_equal(y.cpu().numpy(), want.numpy())
    y, ws = outs[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(y, ws)
    for turn in range(4):
        x2, sx2 = codes(rows, d_in, 10 + turn)
        xd.copy_(on_gpu(x2))
        sxd.copy_(torch.from_numpy(sx2))
        y.zero_()
        graph.replay()
        call(*outs[1])
        torch.cuda.synchronize()
        want = ref.product(x2, w, sx2, sw, None, torch.float32)
        np.testing.assert_array_equal(y.cpu().numpy(), want.numpy())
        np.testing.assert_array_equal(outs[1][0].cpu().numpy(), want.numpy())


def test_refusals(lib):
    need = zipml.row8_product_workspace_bytes(4, 6, 40)
    assert need > 0

    def call(x=FAKE, ldx=48, sx=FAKE, w=FAKE, ldw=48, sw=FAKE, bias=FAKE, rows=4, d_out=6, d_in=40, y=FAKE, dtype=zipml.F32, ldy=6, ws=FAKE,
             n=1 << 30):
        return lib.zipml_row8_product(None, x, ldx, sx, w, ldw, sw, bias, rows, d_out, d_in, y, dtype, ldy, ws, n)
    for kw in ({"x": None}, {"sx": None}, {"w": None}, {"sw": None}, {"y": None}, {"rows": 0}, {"d_out": 0}, {"d_in": 0}, {"rows": -1},
               {"d_out": (1 << 24) + 1, "ldy": 1 << 25}, {"ldx": 40}, {"ldw": 32}, {"ldx": 56}, {"ldx": (1 << 22) + 16}, {"ldw": (1 << 22) + 16},
               {"ldy": 5}, {"dtype": 2}, {"dtype": -1}, {"ldy": 1 << 60}):
        assert call(**kw) == zipml.EINVAL, kw
    assert call(d_in=131072, ldx=131072, ldw=131072) == zipml.ERANGE
    assert zipml.row8_product_workspace_bytes(4, 6, 131072) == zipml.row8_product_workspace_bytes(0, 6, 40) == 0
    assert call(ws=None) == call(n=need - 1) == zipml.EWORKSPACE
    for name in ("x", "w", "y", "ws"):
        assert call(**{name: ODD}) == zipml.EALIGN, name
    assert call(sx=HALF) == call(sw=HALF) == call(bias=HALF) == zipml.EALIGN
