"""Global norm of many gradients and clipping: the norm against 64 bits, every output bit for bit from the factor, norms that are not
finite, tensors in place, and refusals."""
import ctypes as C
import math
import os

import numpy as np
import pytest
import torch

from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD = 0x1000, 0x1002                             # never dereferenced: the checks come first
BF16, F32 = torch.bfloat16, torch.float32
SIZES = [1, 0, 7, 8, 9, 2047, 2048, 8191, 8192, 8193, 3, 100003]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    return zipml.lib()


def gradients(sizes, kinds, seed=0, size=0.02, at=0):
    """Tensors on the GPU, `at` values into an allocation of their own."""
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n + at, generator=g) * size).to(k).to(DEV)[at:] for n, k in zip(sizes, kinds)]


def exact_norm(grads):
    return math.sqrt(math.fsum(math.fsum((t.double().cpu().numpy().ravel() ** 2).tolist()) for t in grads))


def clipped(grads, outs, max_norm):
    n = torch.full((2,), -1.0, device=DEV)
    ws = torch.full((zipml.clip_workspace_bytes(len(grads)),), 0xFF, dtype=torch.uint8, device=DEV)
    zipml.clip(zipml.ClipList(grads, outs), max_norm, n, ws)
    return n.tolist()


def check(grads, outs, max_norm):
    before = [t.float().cpu().clone() for t in grads]
    want = exact_norm(grads)
    norm, factor = clipped(grads, outs, max_norm)
    # one rounding to fp32, and a 64-bit sum in another order
    assert abs(norm - want) <= 2.0 ** -24 * want * (1 + 1e-6)
    by = 1.0 if want <= max_norm else max_norm / want
    assert abs(factor - by) <= 2.0 ** -24 * by * (1 + 1e-6)
    for b, o in zip(before, grads if outs is None else outs):
        if o is not None:
            assert torch.equal(o.cpu(), (b * torch.tensor(factor, dtype=F32)).to(o.dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("at", [0, 1, 3])
@pytest.mark.parametrize("kind,out", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("max_norm", [0.25, 1e6])
def test_norm_and_outputs(kind, out, max_norm, at):
    grads = gradients(SIZES, [kind] * len(SIZES), 1, at=at)
    outs = [torch.full((n + at + 1,), 7.0, dtype=out, device=DEV)[at:at + n] for n in SIZES]
    check(grads, outs, max_norm)
    for o in outs:                                     # the value behind each stays
        whole = torch.as_strided(o, (o.numel() + 1,), (1,))
        assert float(whole[-1]) == 7.0


@pytest.mark.gpu
@pytest.mark.parametrize("max_norm", [0.25, 1e6, 0.0])
def test_in_place_and_without_output(max_norm):
    kinds = [F32, BF16] * (len(SIZES) // 2)
    check(gradients(SIZES, kinds, 2), None, max_norm)
    grads = gradients(SIZES, kinds, 3)
    kept = [t.clone() for t in grads]
    check(grads, [None if k % 2 else t for k, t in enumerate(grads)], max_norm)
    for k, (a, b) in enumerate(zip(grads, kept)):
        if k % 2:
            assert torch.equal(a, b)
    check(grads, [None] * len(grads), max_norm)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [64, 65, 128, 129, 160, 161, 500])
def test_many_tensors(n):
    """As many as the lanes of a wave, as a launch takes, and more."""
    sizes = [(37 * k) % 5000 for k in range(n)]
    grads = gradients(sizes, [F32 if k % 3 else BF16 for k in range(n)], 4)
    bucket = torch.empty(sum(sizes), dtype=BF16, device=DEV)
    check(grads, list(bucket.split(sizes)), 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("n,size", [(320, 20001), (330, 20001), (700, 16389), (3001, 300)])
def test_many_tensors_with_many_sums(n, size):
    grads = gradients([size - k % 3 for k in range(n)], [F32] * n, seed=n)
    check(grads, [torch.empty_like(t, dtype=BF16) if k % 7 else None for k, t in enumerate(grads)], 0.5)
    check(grads, None, 0.5)


@pytest.mark.gpu
def test_many_values():
    """More chunks than workgroups."""
    grads = gradients([9_000_001, 5, 4_000_000], [F32, BF16, BF16], 5)
    check(grads, [torch.empty_like(t, dtype=F32) for t in grads], 1.0)


@pytest.mark.gpu
def test_a_tensor_of_more_than_2_to_the_32_values():
    """Offsets and chunks past 32 bits: the bits of values at its end, and the norm (all squares are 1/4: exact)."""
    n = (1 << 32) + 5000
    big, out = torch.full((n,), 0.5, dtype=BF16, device=DEV), torch.empty(n, dtype=BF16, device=DEV)
    big[-3:] = 2.0
    norm, factor = clipped([torch.ones(7, device=DEV), big], [None, out], 256.0)
    want = math.sqrt(7 + (n - 3) / 4 + 12)
    assert abs(norm - want) <= 2.0 ** -24 * want and abs(factor - 256.0 / want) <= 2.0 ** -23 * factor
    ends = torch.cat([out[:4], out[(1 << 32) - 4:(1 << 32) + 4], out[-4:]]).float().cpu()
    small, large = (float(torch.tensor(v * factor, dtype=F32).to(BF16)) for v in (0.5, 2.0))
    assert ends.tolist() == [small] * 13 + [large] * 3


@pytest.mark.gpu
def test_large_and_small_values():
    """Squares that fp32 does not hold."""
    check(gradients([5000, 300], [F32, F32], 6, 1e30), None, 1.0)
    check(gradients([5000, 300], [F32, F32], 7, 1e-30), None, 1e-28)


@pytest.mark.gpu
def test_norms_that_are_not_finite():
    grads = gradients([100, 200], [F32, F32], 8)
    grads[0][5] = float("inf")
    norm, factor = clipped(grads, None, 1.0)
    assert norm == math.inf and factor == 0.0
    assert torch.isnan(grads[0]).sum() == 1 and torch.isnan(grads[0][5]) and (grads[1] == 0).all()
    grads = gradients([100, 200], [F32, F32], 9)
    grads[1][7] = float("nan")
    norm, factor = clipped(grads, None, 1.0)
    assert math.isnan(norm) and math.isnan(factor) and all(torch.isnan(t).all() for t in grads)
    grads = gradients([100], [F32], 10, 0.0)
    assert clipped(grads, None, 0.0) == [0.0, 1.0]


@pytest.mark.gpu
def test_in_a_graph():
    grads = gradients([3000, 70000, 11], [F32, BF16, F32], 11)
    outs = [torch.empty_like(t) for t in grads]
    n, ws = torch.empty(2, device=DEV), torch.empty(zipml.clip_workspace_bytes(3), dtype=torch.uint8, device=DEV)
    tensors = zipml.ClipList(grads, outs)
    zipml.clip(tensors, 0.5, n, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zipml.clip(tensors, 0.5, n, ws)
    for turn in range(4):
        for t, new in zip(grads, gradients([3000, 70000, 11], [F32, BF16, F32], 20 + turn)):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs] + [n.clone()]
        zipml.clip(tensors, 0.5, n, ws)
        assert all(torch.equal(a, b) for a, b in zip(got, outs + [n]))
        assert abs(float(n[0]) - exact_norm(grads)) <= 2.0 ** -23 * float(n[0])


# ---- refusals ---------------------------------------------------------------------------------

def entry(grad=FAKE, out=FAKE, count=8, gd=zipml.F32, od=zipml.F32):
    return zipml._ClipTensor(grad, out, count, gd, od)


def test_refusals(lib):
    def call(*entries, n=None, tensors=True, max_norm=1.0, norm=C.c_void_p(FAKE), ws=C.c_void_p(FAKE), size=1 << 20):
        table = (zipml._ClipTensor * max(1, len(entries)))(*entries)
        return lib.zipml_clip(None, table if tensors else None, len(entries) if n is None else n, max_norm, norm, ws, size)
    ok = entry()
    for kw in ({"n": 0}, {"n": -1}, {"n": (1 << 20) + 1}, {"tensors": False}, {"max_norm": -1.0}, {"max_norm": float("nan")}, {"norm": None}):
        assert call(ok, **kw) == zipml.EINVAL, kw
    for bad in (entry(gd=2), entry(od=-1), entry(count=-1), entry(count=(1 << 33) + 1), entry(grad=None), entry(od=zipml.BF16)):
        assert call(ok, bad) == zipml.EINVAL
    assert call(ok, ws=None) == call(ok, size=zipml.clip_workspace_bytes(1) - 1) == zipml.EWORKSPACE
    assert call(ok, entry(grad=ODD)) == call(ok, entry(out=ODD)) == zipml.EALIGN
    assert call(ok, ws=C.c_void_p(0x1004)) == call(ok, norm=C.c_void_p(ODD)) == zipml.EALIGN
    assert zipml.clip_workspace_bytes(0) == zipml.clip_workspace_bytes((1 << 20) + 1) == 0


def test_lists_that_are_refused():
    a, b = torch.zeros(40), torch.zeros(40)
    wide = torch.zeros(10, 8)
    for grads, outs in (([], None), ([a], [b, b]), ([a], [torch.zeros(39)]), ([wide[:, :4]], None), ([a.double()], None), ([a, b], [a, a]),
                        ([a, a], None), ([a, b], [b, a]), ([a[:20], b], [a[10:30], b]), ([a, b], [b[:40], None]), ([a], [a.half()])):
        with pytest.raises(zipml.ZipmlError) as e:
            zipml.ClipList(grads, outs)
        assert e.value.code == zipml.EINVAL
    for grads, outs in (([a, b], None), ([a, b], [None, b]), ([a, a], [None, b]), ([a, b], [torch.zeros(40), torch.zeros(40, dtype=BF16)]),
                        ([a[:0], a], None), ([a[:20], a[20:]], None)):
        assert len(zipml.ClipList(grads, outs).table) == 2
