"""Root-mean-square norm with the residual's addition: what it writes bit for bit against the definition, its backward pass against the
formula in 64 bits and against differences, rows that are not finite, outputs in the place of inputs, and refusals."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import row8_reference as ref
from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD, HALF = C.c_void_p(0x1000), C.c_void_p(0x1004), C.c_void_p(0x1002)     # never dereferenced: the checks come first
OTHER, THIRD = C.c_void_p(0x2000), C.c_void_p(0x3000)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SIZES = [(1, 1, 0), (1, 2048, 0), (3, 15, 1), (5, 16, 0), (7, 17, 2), (2, 64, 8), (130, 70, 5), (64, 1021, 3), (1000, 8, 0), (9, 2056, 8),
         (33, 4104, 0), (3, 9001, 1), (2, 16392, 0), (3, 33000, 5), (1100, 520, 0), (4500, 24, 0), (601, 200, 3), (515, 255, 0), (17, 128, 1), (16500, 130, 0), (16399, 9, 0)]
EPS = 1e-6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    return zipml.lib()


def rows_of(rows, cols, seed, kind, size=1.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(0.7 * rng.standard_normal((1, cols))) * size
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[kind])


def apart(t, ld, fill=float("nan")):
    """Rows ld apart on the GPU, `fill` between them."""
    wide = torch.full((t.shape[0], ld), fill, dtype=t.dtype)
    wide[:, :t.shape[1]] = t
    return wide.to(DEV)


def gain_of(cols, seed=5):
    return 1.0 + 0.2 * np.random.default_rng(seed).standard_normal(cols).astype(np.float32)


def equal(got, want):
    np.testing.assert_array_equal(got.float().cpu().numpy() if isinstance(got, torch.Tensor) else got,
                                  want.float().numpy() if isinstance(want, torch.Tensor) else want)


def forward(x, add, gain, pad, eps=EPS, want=("sum", "y", "codes", "rstd")):
    """Outputs of the library by name, whose surroundings it has to leave alone."""
    rows, cols = x.shape
    ld, kw, out = cols + pad, {}, {}
    if add is not None:
        kw.update(add=apart(add, ld + 1), ldadd=ld + 1)
    if gain is not None:
        kw.update(gain=torch.from_numpy(gain).to(DEV))
    for name, at in (("sum", ld + 2), ("y", ld + 3)):
        if name in want:
            out[name] = torch.full((rows, at), 7.0, dtype=x.dtype, device=DEV)
            kw.update({name: out[name], "ld" + name: at})
    if "codes" in want:
        out["codes"] = torch.full((rows, ref.pitch(cols) + 16), 77, dtype=torch.int8, device=DEV)
        out["scales"] = torch.full((rows + 1,), 5.0, device=DEV)
        kw.update(codes=out["codes"], ldc=ref.pitch(cols) + 16, scales=out["scales"])
    if "rstd" in want:
        out["rstd"] = kw["rstd"] = torch.full((rows + 1,), 5.0, device=DEV)
    zipml.norm_forward(apart(x, ld), ld, rows, cols, eps, **kw)
    for name in ("sum", "y"):
        if name in out:
            assert (out[name][:, cols:] == 7.0).all()
            out[name] = out[name][:, :cols]
    if "codes" in out:
        assert (out["codes"][:, ref.pitch(cols):] == 77).all()
        out["codes"] = out["codes"][:, :ref.pitch(cols)].cpu().numpy()
    for name in ("scales", "rstd"):
        if name in out:
            assert out[name][rows] == 5.0
            out[name] = out[name][:rows].cpu().numpy()
    return out


def same(x, add, gain, pad, eps=EPS, **kw):
    r, rstd, v = ref.norm(x, add, gain, eps)
    got = forward(x, add, gain, pad, eps, **kw)
    c, s = ref.encode(v)
    for name, want in (("sum", r), ("rstd", rstd), ("y", torch.from_numpy(v).to(x.dtype)), ("scales", s), ("codes", c)):
        if name in got:
            equal(got[name], want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", SIZES)
def test_all_outputs(kind, rows, cols, pad):
    same(rows_of(rows, cols, 1, kind), rows_of(rows, cols, 2, kind, 2.0), gain_of(cols), pad)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [40, 2500, 40000])
@pytest.mark.parametrize("want", [("y",), ("codes",), ("sum", "codes"), ("y", "rstd"), ("codes", "rstd")])
def test_outputs_that_are_not_wanted(kind, cols, want):
    for add, gain in ((None, None), (None, gain_of(cols)), (rows_of(9, cols, 2, kind), None)):
        same(rows_of(9, cols, 1, kind), add, gain, 0, want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_sizes_of_values(kind):
    """Rows of zeros, of the smallest and of the largest values, with and without eps."""
    x = rows_of(8, 70, 3, kind)
    for r, size in enumerate([0.0, 1e-38, 1e-20, 1e18, 1e30, 3e37, 1.0, 1e-4]):
        x[r] = (x[r].float() / x[r].float().abs().max() * size).to(x.dtype)
    same(x, None, gain_of(70), 0)
    same(x, None, gain_of(70), 3, eps=0.25)
    same(x[1:], None, None, 0, eps=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("cols", [96, 3000, 40000])
def test_rows_that_are_not_finite(kind, cols):
    """They do not touch the other rows, and their codes decode to NaN throughout."""
    x = rows_of(6, cols, 1, kind)
    x[0, 3], x[2, cols - 1], x[4, 64] = float("nan"), float("-inf"), float("inf")
    got = forward(x, None, None, 0)
    for r in range(6):
        assert np.isnan(got["scales"][r]) == (r in (0, 2, 4)) and (got["codes"][r] == 0).all() == (r in (0, 2, 4))
        assert bool(torch.isfinite(got["y"][r]).all()) == (r not in (0, 2, 4))
    keep = [1, 3, 5]
    alone = forward(x[keep], None, None, 0)
    for name in ("y", "sum"):
        equal(got[name][keep].cpu(), alone[name].cpu())
    np.testing.assert_array_equal(got["codes"][keep], alone["codes"])


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [100, 5000, 40000])
def test_sum_and_result_in_the_place_of_inputs(cols):
    x, add, gain = rows_of(37, cols, 1, "bf16"), rows_of(37, cols, 2, "bf16"), gain_of(cols)
    r, rstd, v = ref.norm(x, add, gain, EPS)
    y = torch.from_numpy(v).to(torch.bfloat16)
    g = torch.from_numpy(gain).to(DEV)
    c, s = ref.encode(v)
    for total, out in (("x", None), ("add", None), (None, "x"), (None, "add"), ("x", "add"), ("add", "x")):
        at = {"x": x.to(DEV), "add": add.to(DEV)}
        codes, scales = torch.zeros(37, ref.pitch(cols), dtype=torch.int8, device=DEV), torch.zeros(37, device=DEV)
        zipml.norm_forward(at["x"], cols, 37, cols, EPS, gain=g, add=at["add"], ldadd=cols, sum=at.get(total), ldsum=cols,
                           y=at.get(out), ldy=cols, codes=codes, ldc=ref.pitch(cols), scales=scales)
        if total:
            equal(at[total], r)
        if out:
            equal(at[out], y)
        equal(codes.cpu().numpy(), c)
        equal(scales, s)


# ---- backward ---------------------------------------------------------------------------------

def backward(dy, r, rstd, gain, dsum, pad, flags=0, dgain=None, want_dgain=True):
    rows, cols = dy.shape
    ld, kw = cols + pad, {}
    if gain is not None:
        kw["gain"] = torch.from_numpy(gain).to(DEV)
    if dsum is not None:
        kw.update(dsum=apart(dsum, ld + 3), lddsum=ld + 3)
    dx = torch.full((rows, ld + 2), 7.0, dtype=dy.dtype, device=DEV)
    if want_dgain:
        dgain = torch.full((cols,), float("nan"), device=DEV) if dgain is None else dgain
        kw.update(dgain=dgain, workspace=torch.full((zipml.norm_backward_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device=DEV))
    zipml.norm_backward(apart(dy, ld), ld, apart(r, ld + 1), ld + 1, rows, cols, torch.from_numpy(rstd).to(DEV), dx, ld + 2, flags=flags, **kw)
    assert (dx[:, cols:] == 7.0).all()
    return dx[:, :cols].cpu().double().numpy(), dgain


def check_backward(rows, cols, pad, kind, with_gain=True, with_dsum=True):
    r, dy = rows_of(rows, cols, 1, kind, 2.0), rows_of(rows, cols, 2, kind, 0.02)
    dsum = rows_of(rows, cols, 3, kind, 0.02) if with_dsum else None
    gain = gain_of(cols) if with_gain else None
    _, rstd, _ = ref.norm(r, None, None, EPS)
    dx, dgain = backward(dy, r, rstd, gain, dsum, pad)
    want, want_dgain, off, off_dgain = ref.norm_gradients(dy.float().numpy(), r.float().numpy(), rstd, gain,
                                                          None if dsum is None else dsum.double().numpy())
    assert (np.abs(dx - want) <= 2.0 ** -24 * off + HALF_STEP[kind] * (np.abs(want) + 2.0 ** -24 * off)).all()
    assert (np.abs(dgain.cpu().double().numpy() - want_dgain) <= 2.0 ** -24 * off_dgain).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", SIZES)
def test_gradients(kind, rows, cols, pad):
    check_backward(rows, cols, pad, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("with_gain,with_dsum", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("cols", [70, 3000, 40000])
def test_gradients_without_gain_or_residual(with_gain, with_dsum, cols):
    check_backward(11, cols, 0, "f32", with_gain, with_dsum)


@pytest.mark.gpu
def test_gradients_against_differences():
    """(L(x + h e) - L(x - h e)) / 2h of L = sum(c y) through the forward pass, in fp32: y is off by some 2^-22 of itself, the difference by
    that over h, its third derivative's part by h^2: at h = 2^-7 both are below 2^-12 of the gradients' size (which is about 1)."""
    rows, cols, h = 2, 12, 2.0 ** -7
    x, c, gain = rows_of(rows, cols, 1, "f32"), rows_of(rows, cols, 2, "f32"), gain_of(cols)

    def loss(x, gain):
        return float((forward(x, None, gain, 0, want=("y",))["y"].cpu().double() * c.double()).sum())
    _, rstd, _ = ref.norm(x, None, gain, EPS)
    dx, dgain = backward(c, x, rstd, gain, None, 0)
    for r in range(rows):
        for k in range(cols):
            e = torch.zeros_like(x)
            e[r, k] = h
            assert abs((loss(x + e, gain) - loss(x - e, gain)) / (2 * h) - dx[r, k]) < 0.02
    for k in range(cols):
        e = np.zeros_like(gain)
        e[k] = h
        assert abs((loss(x, gain + e) - loss(x, gain - e)) / (2 * h) - float(dgain[k])) < 0.02


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [40, 2500, 40000])
def test_adding_to_dgain_and_doing_without(cols):
    r, dy = rows_of(50, cols, 1, "bf16"), rows_of(50, cols, 2, "bf16")
    _, rstd, _ = ref.norm(r, None, None, EPS)
    dx, once = backward(dy, r, rstd, None, None, 0)
    start = torch.arange(cols, device=DEV, dtype=torch.float32)
    _, added = backward(dy, r, rstd, None, None, 0, flags=zipml.NORM_ADD, dgain=start.clone())
    assert torch.equal(added, start + once)
    alone, _ = backward(dy, r, rstd, None, None, 0, want_dgain=False)
    np.testing.assert_array_equal(alone, dx)


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [100, 5000, 40000])
def test_dx_in_the_place_of_inputs(cols):
    r, dy, dsum = (rows_of(33, cols, s, "bf16") for s in (1, 2, 3))
    _, rstd, _ = ref.norm(r, None, None, EPS)
    want, _ = backward(dy, r, rstd, None, dsum, 0, want_dgain=False)
    for name in ("r", "dy", "dsum"):
        at = {"r": r.to(DEV), "dy": dy.to(DEV), "dsum": dsum.to(DEV)}
        zipml.norm_backward(at["dy"], cols, at["r"], cols, 33, cols, torch.from_numpy(rstd).to(DEV), at[name], cols, dsum=at["dsum"],
                            lddsum=cols)
        np.testing.assert_array_equal(at[name].cpu().double().numpy(), want)


@pytest.mark.gpu
def test_the_same_bits_every_time():
    r, dy = rows_of(3000, 520, 1, "bf16"), rows_of(3000, 520, 2, "bf16")
    _, rstd, _ = ref.norm(r, None, None, EPS)
    first = backward(dy, r, rstd, None, None, 0)[1]
    for _ in range(3):
        assert torch.equal(backward(dy, r, rstd, None, None, 0)[1], first)


@pytest.mark.gpu
def test_a_row_that_is_not_finite_stays_alone():
    r, dy = rows_of(9, 300, 1, "f32"), rows_of(9, 300, 2, "f32")
    _, rstd, _ = ref.norm(r, None, None, EPS)
    clean, _ = backward(dy, r, rstd, None, None, 0)
    dy[4, 7] = float("nan")
    dx, dgain = backward(dy, r, rstd, None, None, 0)
    assert np.isnan(dx[4]).all()
    keep = [k for k in range(9) if k != 4]
    np.testing.assert_array_equal(dx[keep], clean[keep])
    assert torch.isnan(dgain).cpu().tolist() == [k == 7 for k in range(300)]


@pytest.mark.gpu
def test_rows_far_apart():
    """Offsets past 32 bits."""
    rows, cols, ld = 5, 24, 1 << 30
    x, add = rows_of(rows, cols, 1, "bf16"), rows_of(rows, cols, 2, "bf16")
    r, rstd, v = ref.norm(x, add, None, EPS)
    wide = torch.empty(2, 4 * ld + cols, dtype=torch.bfloat16, device=DEV)
    for k in range(rows):
        wide[0, k * ld:k * ld + cols], wide[1, k * ld:k * ld + cols] = x[k].to(DEV), add[k].to(DEV)
    out = torch.empty(rows, device=DEV)
    zipml.norm_forward(wide[0], ld, rows, cols, EPS, add=add.to(DEV), ldadd=cols, sum=wide[0], ldsum=ld, y=wide[1], ldy=ld, rstd=out)
    equal(out, rstd)
    for k in range(rows):
        equal(wide[0, k * ld:k * ld + cols], r[k])
        equal(wide[1, k * ld:k * ld + cols], torch.from_numpy(v[k]).to(torch.bfloat16))
    total, y = (torch.stack([wide[i, k * ld:k * ld + cols] for k in range(rows)]) for i in (0, 1))
    dx = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    zipml.norm_backward(y, cols, total, cols, rows, cols, out, dx, cols)
    zipml.norm_backward(wide[1], ld, wide[0], ld, rows, cols, out, wide[1], ld)
    equal(torch.stack([wide[1, k * ld:k * ld + cols] for k in range(rows)]), dx.cpu())


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(3, 100), (900, 2047), (4, 40000)])
def test_vectors_among_other_parameters(rows, cols):
    """gain, dgain, scales and rstd begin anywhere in a buffer, and what lies around them stays."""
    x, dy, gain = rows_of(rows, cols, 1, "bf16"), rows_of(rows, cols, 2, "bf16"), gain_of(cols)
    r, rstd, v = ref.norm(x, None, gain, EPS)
    flat = torch.full((2 * cols + 2 * rows + 9,), 7.0, device=DEV)
    g, dg, s, q = flat[1:1 + cols], flat[cols + 2:2 * cols + 2], flat[2 * cols + 3:2 * cols + 3 + rows], flat[2 * cols + rows + 6:2 * cols + 2 * rows + 6]
    g.copy_(torch.from_numpy(gain))
    codes = torch.zeros(rows, ref.pitch(cols), dtype=torch.int8, device=DEV)
    zipml.norm_forward(x.to(DEV), cols, rows, cols, EPS, gain=g, codes=codes, ldc=ref.pitch(cols), scales=s, rstd=q)
    c, want = ref.encode(v)
    equal(codes.cpu().numpy(), c)
    equal(s, want)
    equal(q, rstd)
    ws = torch.empty(zipml.norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    zipml.norm_backward(dy.to(DEV), cols, x.to(DEV), cols, rows, cols, q, torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV), cols, ws,
                        gain=g, dgain=dg)
    _, dgain = backward(dy, x, rstd, gain, None, 0)
    assert torch.equal(dg, dgain)
    rest = torch.ones_like(flat, dtype=torch.bool)
    for t in (g, dg, s, q):
        rest[t.storage_offset():t.storage_offset() + t.numel()] = False
    assert (flat[rest] == 7.0).all() and rest.sum() == 9


# ---- refusals ---------------------------------------------------------------------------------

def test_refusals(lib):
    def fwd(x=FAKE, ldx=40, add=FAKE, ldadd=40, dtype=zipml.BF16, rows=4, cols=40, gain=FAKE, eps=1e-6, total=OTHER, ldsum=40, y=THIRD,
            ldy=40, codes=FAKE, ldc=48, scales=FAKE, rstd=FAKE):
        return lib.zipml_norm_forward(None, x, ldx, add, ldadd, dtype, rows, cols, gain, eps, total, ldsum, y, ldy, codes, ldc, scales, rstd)
    for kw in ({"x": None}, {"ldx": 39}, {"ldadd": 39}, {"ldsum": 39}, {"ldy": 39}, {"ldc": 40}, {"ldc": 32}, {"dtype": 2}, {"rows": 0},
               {"cols": 0}, {"rows": -1}, {"eps": -1e-6}, {"eps": float("nan")}, {"eps": float("inf")}, {"codes": None}, {"scales": None},
               {"y": None, "codes": None, "scales": None}, {"ldx": 1 << 60}, {"ldsum": 1 << 60}, {"cols": 1 << 31, "ldx": 1 << 31},
               # in the place of an input at another pitch, or both results in one place
               {"total": FAKE, "ldsum": 48}, {"y": FAKE, "ldy": 48}, {"add": THIRD, "ldadd": 41}, {"y": OTHER}):
        assert fwd(**kw) == zipml.EINVAL, kw
    for name in ("x", "add", "total", "y", "codes"):
        assert fwd(**{name: ODD}) == zipml.EALIGN, name
    assert fwd(scales=HALF) == fwd(rstd=HALF) == fwd(gain=HALF) == zipml.EALIGN

    need = zipml.norm_backward_workspace_bytes(4, 40)

    def bwd(dy=FAKE, lddy=40, total=FAKE, ldsum=40, dtype=zipml.BF16, rows=4, cols=40, gain=FAKE, rstd=FAKE, dsum=FAKE, lddsum=40, dx=OTHER,
            lddx=40, dgain=FAKE, flags=0, ws=FAKE, n=need):
        return lib.zipml_norm_backward(None, dy, lddy, total, ldsum, dtype, rows, cols, gain, rstd, dsum, lddsum, dx, lddx, dgain, flags, ws, n)
    for kw in ({"dy": None}, {"total": None}, {"rstd": None}, {"dx": None}, {"lddy": 39}, {"ldsum": 39}, {"lddsum": 39}, {"lddx": 39},
               {"dtype": 5}, {"rows": 0}, {"cols": -1}, {"flags": 2}, {"flags": zipml.NORM_ADD, "dgain": None}, {"dx": FAKE, "lddx": 48},
               {"dsum": OTHER, "lddsum": 48}):
        assert bwd(**kw) == zipml.EINVAL, kw
    assert bwd(ws=None) == bwd(n=need - 1) == zipml.EWORKSPACE
    for name in ("dy", "total", "dsum", "dx", "ws"):
        assert bwd(**{name: ODD}) == zipml.EALIGN, name
    assert bwd(rstd=HALF) == bwd(gain=HALF) == bwd(dgain=HALF) == zipml.EALIGN
    assert zipml.norm_backward_workspace_bytes(0, 5) == zipml.norm_backward_workspace_bytes(5, 0) == 0
    assert zipml.norm_backward_workspace_bytes(1 << 20, 1 << 20) <= 1 << 28
