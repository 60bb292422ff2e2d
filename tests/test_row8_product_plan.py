"""Every shape, number of ranges and way of writing that the product on 8-bit codes chooses, bit for bit, each at a size of which the test
first asserts that it is chosen."""
import ctypes as C

import numpy as np
import pytest
import torch

import row8_reference as ref
import test_row8_product as product_test
from paper_1611_05402_amd import zipml

lib = product_test.lib
DEV = "cuda"

# (outputs, tokens, waves) of a tile, ranges, past the caches: rows, d_out, d_in
PATHS = {
    ((16, 16, 4), 1, 0): (5, 131, 333),
    ((16, 16, 8), 1, 0): (3, 201, 700),
    ((16, 16, 16), 1, 0): (3, 201, 2043),
    ((32, 32, 4), 1, 0): (5881, 18, 23),
    ((32, 32, 8), 1, 0): (7930, 3, 524),
    ((32, 32, 16), 1, 0): (374, 423, 1706),
    ((64, 32, 8), 1, 0): (127, 4093, 1030),
    ((64, 64, 8), 1, 0): (1000, 1003, 521),
    ((128, 64, 4), 1, 0): (15363, 35, 70),
    ((128, 64, 4), 3, 0): (33, 9867, 6390),
    ((128, 64, 4), 4, 0): (33, 6091, 10441),
    ((128, 64, 4), 8, 0): (32, 3717, 14547),
    ((128, 128, 8), 1, 0): (1025, 2043, 4100),
    ((128, 128, 8), 1, 1): (16390, 4160, 40),
    ((128, 128, 8), 2, 0): (700, 2557, 10250),
    ((128, 128, 8), 3, 0): (10057, 69, 3318),
    ((128, 128, 8), 4, 0): (301, 2557, 10241),
    ((128, 128, 8), 8, 0): (4022, 19, 16351),
    ((256, 256, 8), 1, 0): (5000, 5121, 1111),
    ((256, 256, 8), 1, 1): (4097, 8128, 1111),
    ((256, 256, 8), 2, 0): (15019, 265, 3727),
    ((256, 256, 8), 3, 0): (2047, 2559, 10247),
    ((256, 256, 8), 4, 0): (11106, 131, 9177),
    ((256, 256, 8), 8, 0): (195, 7035, 18869),
}
# workgroups that stay: one round to each tile, and sums of ranges
PATHS_STAY = [(((256, 256, 8), 1, 1), (16384, 4096, 40)), (((256, 256, 8), 3, 0), (16557, 394, 16826))]
ALL = list(PATHS.items()) + PATHS_STAY


def path(rows, d_out, d_in, dtype=zipml.BF16, ldy=None):
    p = zipml.debug_product_plan(rows, d_out, d_in, dtype, ldy)
    return (p.outputs, p.tokens, p.waves), p.ranges, p.past_caches


def room(rows, d_out, d_in):
    return zipml.row8_product_workspace_bytes(rows, d_out, d_in)


@pytest.mark.parametrize("wanted,sizes", ALL)
def test_sizes_take_their_paths(lib, wanted, sizes):
    for dtype in (zipml.BF16, zipml.F32):
        assert path(*sizes, dtype) == wanted
    rows, d_out, _ = sizes
    (outputs, tokens, _), ranges, past = wanted
    work = -(-d_out // outputs) * -(-rows // tokens) * ranges
    assert zipml.debug_product_plan(*sizes).workgroups == (min(256, work) if outputs == 256 else work)
    # a range's sums: 32 bits for each of a row's outputs, four of them side by side
    assert room(*sizes) == (256 if ranges == 1 else ranges * rows * (-(-d_out // 4) * 4) * 4)
    # rows that do not begin at lines of 128 bytes go through the caches
    assert path(*sizes, zipml.BF16, -(-d_out // 64) * 64 + 8)[2] == 0


def test_the_staying_tiles_follow_one_another():
    """More pieces of work than workgroups, with one round of 128 codes to a tile and with many."""
    for _, (rows, d_out, d_in) in PATHS_STAY + [(None, PATHS[(256, 256, 8), 1, 0]), (None, PATHS[(256, 256, 8), 1, 1])]:
        p = zipml.debug_product_plan(rows, d_out, d_in)
        assert p.workgroups == 256 < -(-d_out // 256) * -(-rows // 256) * p.ranges


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("wanted,sizes", list(PATHS.items()))
def test_bits_on_each_path(wanted, sizes, kind):
    assert path(*sizes, zipml.BF16 if kind == "bf16" else zipml.F32) == wanted
    product_test.same(*sizes, kind, bias=True)


@pytest.mark.gpu
@pytest.mark.parametrize("wanted,sizes", PATHS_STAY)
def test_bits_where_tiles_follow_one_another(wanted, sizes):
    assert path(*sizes) == wanted
    product_test.same(*sizes, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [PATHS[(128, 64, 4), 8, 0], PATHS[(128, 128, 8), 4, 0], PATHS[(256, 256, 8), 3, 0]])
def test_ranges_without_a_bias_to_rows_apart(sizes):
    assert path(*sizes, zipml.F32, sizes[1] + 5)[1] > 1
    product_test.same(*sizes, "f32", more=32, pad=5)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [PATHS[(128, 64, 4), 8, 0], PATHS[(128, 128, 8), 4, 0], PATHS[(256, 256, 8), 3, 0]])
def test_ranges_on_two_streams_and_in_two_graphs(sizes):
    """Each stream with a workspace of its own, two graphs with one; every one of them holds sums."""
    rows, d_out, d_in = sizes
    assert path(*sizes)[1] > 1 and room(*sizes) > 256
    product_test.test_two_streams_at_once_and_a_graph(rows, d_out, d_in)
    (w, sw), ws = product_test.codes(d_out, d_in, 2), torch.empty(room(*sizes), dtype=torch.uint8, device=DEV)
    wd, swd = product_test.on_gpu(w), torch.from_numpy(sw).to(DEV)
    inputs = [[product_test.on_gpu(x), torch.from_numpy(s).to(DEV)] for x, s in (product_test.codes(rows, d_in, k) for k in (1, 5))]
    outs, graphs = [torch.empty(rows, d_out, device=DEV) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]

    def call(k, y=None):
        x, s = inputs[k]
        zipml.row8_product(x, x.stride(0), s, wd, wd.stride(0), swd, rows, d_out, d_in, outs[k] if y is None else y, d_out, ws)
    call(0)
    torch.cuda.synchronize()
    for k in range(2):
        with torch.cuda.graph(graphs[k]):
            call(k)
    for turn in range(3):
        wants = []
        for k in range(2):
            x, s = product_test.codes(rows, d_in, 20 + 2 * turn + k)
            inputs[k][0].copy_(product_test.on_gpu(x))
            inputs[k][1].copy_(torch.from_numpy(s))
            wants.append(ref.product(x, w, s, sw, None, torch.float32))
        for k in (turn % 2, 1 - turn % 2):
            outs[k].zero_()
            graphs[k].replay()
        torch.cuda.synchronize()
        eager = torch.empty(rows, d_out, device=DEV)
        call(0, eager)
        for got, want in ((outs[0], wants[0]), (outs[1], wants[1]), (eager, wants[0])):
            np.testing.assert_array_equal(got.cpu().numpy(), want.numpy())


def test_refusals(lib):
    plan = zipml.ProductPlan()

    def call(rows=4, d_out=6, d_in=40, dtype=zipml.F32, ldy=6, size=256, out=C.byref(plan)):
        return lib.zipml_debug_product_plan(rows, d_out, d_in, dtype, ldy, size, out)
    assert call() == zipml.OK
    for kw in ({"rows": 0}, {"d_out": 0}, {"d_in": 0}, {"dtype": 2}, {"ldy": 5}, {"ldy": 1 << 60}, {"out": None}, {"d_out": (1 << 24) + 1, "ldy": 1 << 25}):
        assert call(**kw) == zipml.EINVAL, kw
    assert call(d_in=131072) == zipml.ERANGE
    assert call(size=255) == call(size=0) == zipml.EWORKSPACE


@pytest.mark.parametrize("rows,d_out,d_in", [(1 << 28, 8, 16), ((1 << 28) - 16, 8, 16), (1 << 27, 8, 600), (1 << 27, 16, 600), (1 << 26, 3, 2000),
                                             (1 << 31, 1, 1), (1 << 31, 512, 16), ((1 << 31) - 255, 300, 1), (1 << 30, 1024, 100), (1 << 16, 1 << 24, 16),
                                             (1 << 20, 1 << 20, 131071), (1 << 29, 40, 131071), (7, 1 << 24, 131071), ((1 << 27) + 1, 17, 200)])
def test_launches_of_all_sizes_fit(lib, rows, d_out, d_in):
    """A launch holds fewer than 2^32 threads."""
    p = zipml.debug_product_plan(rows, d_out, d_in)
    assert 0 < p.workgroups * p.waves * 64 < 1 << 32
    assert p.ranges == 1 and room(rows, d_out, d_in) == 256


@pytest.mark.gpu
@pytest.mark.parametrize("rows,d_out", [(1 << 28, 8), (1 << 31, 3)])
def test_more_rows_than_a_launch_of_the_smallest_tiles_holds(rows, d_out):
    """Up to the largest number of tokens, all results compared (an elementwise chain of single fp32 operations on exact sums, below 2^24 and so
    exact in fp32)."""
    d_in, piece = 16, 1 << 24
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randint(-127, 128, (rows // 64, d_in), generator=g, device=DEV, dtype=torch.int8).repeat(64, 1)
    w = torch.randint(-127, 128, (d_out, d_in), generator=g, device=DEV, dtype=torch.int8)
    sx, sw = torch.rand(rows, generator=g, device=DEV), torch.rand(d_out, generator=g, device=DEV)
    y = torch.full((rows + 1, d_out), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(room(rows, d_out, d_in), dtype=torch.uint8, device=DEV)
    zipml.row8_product(x, d_in, sx, w, d_in, sw, rows, d_out, d_in, y, d_out, ws)
    for r in range(0, rows, piece):
        sums = torch.mm(x[r:r + piece].float(), w.float().t().contiguous())
        assert torch.equal(y[r:r + piece], (sums * sx[r:r + piece, None] * sw).to(torch.bfloat16)), r
    assert (y[rows] == 7.0).all()


RANGED = [s for (_, ranges, _), s in PATHS.items() if ranges > 1]


@pytest.mark.parametrize("sizes", RANGED)
def test_less_room_takes_fewer_ranges(lib, sizes):
    rows, d_out, d_in = sizes
    need, sums = room(*sizes), rows * (-(-d_out // 4) * 4) * 4
    most = zipml.debug_product_plan(*sizes).ranges
    for size in (256, sums, 2 * sums, need - 1, need, need + 1, 1 << 40):
        p = zipml.debug_product_plan(*sizes, workspace_bytes=max(256, size))
        assert p.ranges == 1 or p.ranges * sums <= size
        assert (p.ranges == most) == (size >= need)
    # the call itself gets past its check of the room (and refuses x, whose address is no multiple of 16)
    ok, odd = C.c_void_p(0x1000), C.c_void_p(0x1004)
    ldx = -(-d_in // 16) * 16
    for size, code in ((256, zipml.EALIGN), (need - 1, zipml.EALIGN), (255, zipml.EWORKSPACE)):
        assert lib.zipml_row8_product(None, odd, ldx, ok, ok, ldx, ok, None, rows, d_out, d_in, ok, zipml.BF16, d_out, ok, size) == code


@pytest.mark.gpu
def test_the_room_of_one_batch_serves_others():
    """Of 10,240 -> 2,560, whose need falls and rises with the rows: each call with the room that another number of rows asks for, which
    leaves what lies behind it as it is."""
    d_out, d_in, all_rows = 2560, 10240, (300, 1024, 700, 2048)
    (x, sx), (w, sw) = product_test.codes(2048, d_in, 1), product_test.codes(d_out, d_in, 2)
    xd, wd, sxd, swd = product_test.on_gpu(x), product_test.on_gpu(w), torch.from_numpy(sx).to(DEV), torch.from_numpy(sw).to(DEV)
    want = ref.product(x, w, sx, sw, None, torch.float32)
    needs = sorted({room(r, d_out, d_in) for r in all_rows} | {room(300, d_out, d_in) - 1})
    assert needs[0] == 256 < needs[1] < needs[-1]
    for need in needs:
        ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
        for rows in all_rows:
            y = torch.full((rows, d_out), float("nan"), device=DEV)
            zipml.row8_product(xd, d_in, sxd, wd, d_in, swd, rows, d_out, d_in, y, d_out, ws[:need])
            np.testing.assert_array_equal(y.cpu().numpy(), want[:rows].numpy())
            assert (ws[need:] == 0xA5).all()
