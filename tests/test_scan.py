"""The gated recurrence: forward, stored inputs, backward and single tokens, against the definition in 64 bits."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import act_reference as act
import scan_reference as ref
from paper_1611_05402_amd import zipml

DEV = "cuda"
FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -23}              # of a result that is rounded once


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(zipml.LIB_PATH):
        from paper_1611_05402_amd import build
        build.build()
    return zipml.lib()


def host(t):
    return t.double().cpu().numpy()


def offsets(name, tokens):
    return {"one": [0, tokens],
            "empty ones": [0, 0, tokens // 3, tokens // 3, tokens // 3, tokens, tokens],
            "filled up": [min(2, tokens - 1), tokens // 2, max(tokens // 2, tokens - 3)],
            "single tokens": list(range(tokens + 1)),
            "no token": [0, 0, 0],
            "nowhere": [tokens, tokens]}[name]


class Problem:
    """x and z side by side in rows of a wider tensor whose other columns are NaN."""

    def __init__(self, tokens, channels, start, kind, pad=0, seed=0, scale_z=1.5, mean_z=2.0):
        rng = np.random.default_rng(seed + tokens * 3 + channels)
        self.tokens, self.channels, self.kind, self.start = tokens, channels, kind, np.asarray(start, np.int64)
        self.n = len(start) - 1
        self.zat = -(-channels // 8) * 8
        self.ld = self.zat + channels + pad
        w = torch.full((tokens, self.ld), float("nan"), dtype=TYPES[kind])
        w[:, :channels] = torch.from_numpy(rng.standard_normal((tokens, channels))).to(TYPES[kind])
        w[:, self.zat:self.zat + channels] = torch.from_numpy(
            rng.standard_normal((tokens, channels)) * scale_z + mean_z).to(TYPES[kind])
        self.set(w)
        self.h0 = torch.from_numpy(rng.standard_normal((self.n, channels)).astype(np.float32)).to(DEV)
        self.dy = torch.from_numpy(rng.standard_normal((tokens, channels)).astype(np.float32)).to(TYPES[kind]).to(DEV)
        self.dh_last = torch.from_numpy(rng.standard_normal((self.n, channels)).astype(np.float32)).to(DEV)
        self.start_dev = torch.from_numpy(self.start).to(DEV)
        self.ws = torch.full((zipml.scan_workspace_bytes(tokens, channels),), 0xFF, dtype=torch.uint8, device=DEV)

    def set(self, w):
        self.w = w.to(DEV)
        self.x, self.z = self.w[:, :self.channels], self.w[:, self.zat:self.zat + self.channels]

    def new(self, *shape, dtype=None):
        return torch.full(shape, 9.0, dtype=dtype or torch.float32, device=DEV)

    def forward(self, train=False, h0=True, seq=True, last=True, seed=5, epoch=3, tag=7):
        t, c = self.tokens, self.channels
        self.ybuf = self.new(t, c + 5, dtype=TYPES[self.kind])
        self.last = self.new(self.n, c) if last else None
        kw = {}
        if train:
            self.ax, self.az = (torch.full((zipml.act_bytes(t, c),), 0xCD, dtype=torch.uint8, device=DEV) for _ in range(2))
            self.states = self.new(-(-t // 256), c)
            kw = dict(act_x=self.ax, act_z=self.az, states=self.states, seed=seed, epoch=epoch, tag=tag)
        zipml.scan_forward(self.x, self.ld, self.z, self.ld, t, c, self.ybuf, c + 5, self.ws,
                           seq_start=self.start_dev if seq else None, n_seq=self.n, h0=self.h0 if h0 else None,
                           h_last=self.last, **kw)
        assert (self.ybuf[:, c:] == 9.0).all()
        return self.ybuf[:, :c]

    def backward(self, h0=True, seq=True, dh_last=True, dh0=True):
        t, c = self.tokens, self.channels
        g = self.new(t, self.ld + 1, dtype=TYPES[self.kind])
        self.dh0 = self.new(self.n, c) if dh0 else None
        zipml.scan_backward(self.ax, self.az, self.states, self.dy, c, t, c, g, self.ld + 1, g[:, self.zat:], self.ld + 1,
                            self.ws, seq_start=self.start_dev if seq else None, n_seq=self.n,
                            h0=self.h0 if h0 else None, dh_last=self.dh_last if dh_last else None, dh0=self.dh0)
        assert (g[:, c:self.zat] == 9.0).all() and (g[:, self.zat + c:] == 9.0).all()
        return g[:, :c], g[:, self.zat:self.zat + c]

    def h0_host(self, used=True):
        return host(self.h0) if used else np.zeros((self.n, self.channels))


def close(got, want, off, kind):
    assert (np.abs(host(got) - want) <= off + ROUND[kind] * np.abs(want) + 1e-30).all()


SHAPES = [(1, 1, "one"), (1, 64, "one"), (2, 70, "single tokens"), (7, 8, "empty ones"), (255, 31, "one"),
          (256, 65, "empty ones"), (257, 130, "one"), (600, 3, "filled up"), (300, 40, "single tokens"),
          (1029, 96, "empty ones"), (5, 16, "no token"), (300, 9, "nowhere"), (2500, 17, "one")]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,channels,seqs", SHAPES)
def test_forward(kind, tokens, channels, seqs):
    for pad in (0, 3):
        p = Problem(tokens, channels, offsets(seqs, tokens), kind, pad)
        y = p.forward()
        want, last, off, last_off = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
        close(y, want, off, kind)
        close(p.last, last, last_off, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,channels,seqs", SHAPES)
def test_training_step(kind, tokens, channels, seqs):
    for pad in (0, 3):
        p = Problem(tokens, channels, offsets(seqs, tokens), kind, pad)
        y = p.forward(train=True)
        want, last, off, last_off = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
        close(y, want, off, kind)
        close(p.last, last, last_off, "f32")
        for b in range(1, -(-tokens // 256)):
            close(p.states[b], want[256 * b - 1], off[256 * b - 1], "f32")
        qx = act.encode(p.x.float().cpu().numpy(), 5, 3, 7)
        qz = act.encode(np.clip(p.z.float().cpu().numpy(), -16, 16), 5, 3, 8)
        np.testing.assert_array_equal(p.ax.cpu().numpy(), act.pack(*qx))
        np.testing.assert_array_equal(p.az.cpu().numpy(), act.pack(*qz))
        dx, dz = p.backward()
        g, o = ref.backward(act.decode(*qx, channels), act.decode(*qz, channels), want, off, p.start, p.h0_host(),
                            host(p.dy), host(p.dh_last))
        close(dx, g[0], o[0], kind)
        close(dz, g[1], o[1], kind)
        close(p.dh0, g[2], o[2], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 300])
def test_without_the_optional_arrays(tokens):
    """One sequence without offsets, from the zero state; gradients of the outputs alone."""
    p = Problem(tokens, 40, [0, tokens], "f32")
    p.h0.zero_()
    p.dh_last.zero_()
    a, (ax, az) = p.forward(train=True), p.backward()
    b = p.forward(train=True, h0=False, seq=False, last=False)
    bx, bz = p.backward(h0=False, seq=False, dh_last=False, dh0=False)
    assert torch.equal(a, b) and torch.equal(ax, bx) and torch.equal(az, bz)
    assert torch.equal(a, p.forward(h0=False, seq=False, last=False))           # serving gives what training gives


@pytest.mark.gpu
@pytest.mark.parametrize("n", [600, 3000])
def test_many_sequences(n):
    """More sequences than threads, and so many that a block searches for its first, of 0 to 7 tokens each."""
    lengths = np.random.default_rng(2).integers(0, 8, n)
    lengths[n // 2:n // 2 + 90] = 0
    start = np.concatenate([[0], np.cumsum(lengths)])
    p = Problem(int(start[-1]), 20, start, "f32")
    y = p.forward(train=True)
    want, last, off, last_off = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
    close(y, want, off, "f32")
    close(p.last, last, last_off, "f32")
    dx, dz = p.backward()
    qx = act.decode(*act.encode(p.x.cpu().numpy(), 5, 3, 7), 20)
    qz = act.decode(*act.encode(np.clip(p.z.cpu().numpy(), -16, 16), 5, 3, 8), 20)
    g, o = ref.backward(qx, qz, want, off, p.start, p.h0_host(), host(p.dy), host(p.dh_last))
    close(dx, g[0], o[0], "f32")
    close(dz, g[1], o[1], "f32")
    close(p.dh0, g[2], o[2], "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_long_sequence(kind):
    p = Problem(40000, 12, [0, 17, 39990], kind, mean_z=4.0)
    y = p.forward()
    want, last, off, last_off = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
    close(y, want, off, kind)
    close(p.last, last, last_off, "f32")


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_gates_that_are_saturated(kind):
    """z at both infinities, at the type's lowest and highest values and beyond the clamp: closed gates forget, open
    ones hold; the stored z is clamped and its gradients stay finite."""
    p = Problem(700, 64, [0, 700], kind)
    w = p.w.cpu()
    big = torch.finfo(TYPES[kind]).max
    for k, v in enumerate([float("inf"), float("-inf"), big, -big, 40.0, -40.0, 17.0, -17.0]):
        w[:, p.zat + 8 * k] = v
        w[k::11, p.zat + 3] = v
    p.set(w)
    y = p.forward(train=True)
    want, last, off, last_off = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
    close(y, want, off, kind)
    dx, dz = p.backward()
    qx = act.decode(*act.encode(p.x.float().cpu().numpy(), 5, 3, 7), 64)
    qz = act.decode(*act.encode(np.clip(p.z.float().cpu().numpy(), -16, 16), 5, 3, 8), 64)
    g, o = ref.backward(qx, qz, want, off, p.start, p.h0_host(), host(p.dy), host(p.dh_last))
    close(dx, g[0], o[0], kind)
    close(dz, g[1], o[1], kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_nan_and_infinity_stay_in_their_sequence(kind):
    """A NaN reaches every later state of its own sequence and channel, through blocks whose gates multiply to
    nothing, and nothing else; so do tokens that belong to no sequence."""
    tokens, start = 2000, [3, 900, 900, 1500, 1990]
    p = Problem(tokens, 64, start, kind, scale_z=0.1, mean_z=0.0)               # f near 1/2
    clean = host(p.forward())
    w = p.w.cpu()
    w[100, 5] = float("nan")
    w[200, p.zat + 40] = float("nan")
    w[0:3] = float("nan")
    w[1990:] = float("inf")
    p.set(w)
    y = host(p.forward(train=True))
    bad = np.zeros_like(clean, bool)
    bad[100:900, 5] = bad[200:900, 40] = True
    assert np.isnan(y[bad]).all()
    np.testing.assert_array_equal(y[~bad], clean[~bad])
    assert np.isfinite(host(p.last)[1:]).all() and np.isnan(host(p.last)[0, 5])
    dx, dz = (host(v) for v in p.backward())
    for v in (dx, dz):
        assert np.isfinite(v[900:]).all() and (v[:3] == 0).all() and (v[1990:] == 0).all()
    assert np.isfinite(host(p.dh0)[1:]).all()
    assert np.isnan(dz[101:900, 5]).all() and np.isfinite(np.delete(dx, np.s_[32:64], 1)).all()


@pytest.mark.gpu
def test_offsets_that_make_no_sense_touch_nothing_else():
    """Undefined results, but everything outside the arrays stays as it was (the guards are in Problem)."""
    for start in ([0, 500, 100, 400], [-70, 20, 9000], [400, 0], [1 << 40, -(1 << 40), 7]):
        p = Problem(400, 24, [0, 10, 20, 30][:len(start)], "f32")
        p.start_dev = torch.tensor(start, dtype=torch.int64, device=DEV)
        p.forward(train=True)
        p.backward()
        torch.cuda.synchronize()


def on_grid(tokens, channels, seed):
    """fp32 values that 8 bits hold exactly: multiples of 2^-6, the largest of each group 127 * 2^-6."""
    rng = np.random.default_rng(seed)
    v = rng.integers(-127, 128, (tokens, channels)) / 64.0
    v[:, ::32] = 127.0 / 64.0
    return v.astype(np.float32)


@pytest.mark.gpu
def test_gradients_against_differences():
    """Inputs that storage does not change: the backward pass against central differences of the library's own
    forward pass along random directions.  Step 2^-7: the cubic term is below 2^-14 * 0.1 |L'''| and L is a
    sum of 64 x 300 terms of size 1 kept to 2^-24 each, so 2e-3 of the gradient's norm is allowed."""
    tokens, c = 300, 64
    p = Problem(tokens, c, [0, 130, 130, 300], "f32")
    w = p.w.cpu()
    w[:, :c], w[:, p.zat:p.zat + c] = torch.from_numpy(on_grid(tokens, c, 1)), torch.from_numpy(on_grid(tokens, c, 2))
    p.set(w)
    p.forward(train=True)
    dx, dz = p.backward()
    base = p.w.clone()
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)

    def loss():
        y = p.forward()
        return float((y.double() * p.dy.double()).sum() + (p.last.double() * p.dh_last.double()).sum())
    step = 2.0 ** -7
    for grad, at in ((dx, 0), (dz, p.zat)):
        norm = float(grad.double().norm())
        for _ in range(3):
            v = torch.randn(tokens, c, generator=gen, device=DEV)
            values = []
            for sign in (1, -1):
                w = base.clone()
                w[:, at:at + c] += sign * step * v
                p.set(w)
                values.append(loss())
            p.set(base)
            slope = (values[0] - values[1]) / (2 * step)
            assert abs(slope - float((grad.double() * v.double()).sum())) <= 2e-3 * norm
    h0 = p.h0.clone()
    for _ in range(3):
        v = torch.randn(p.n, c, generator=gen, device=DEV)
        values = []
        for sign in (1, -1):
            p.h0 = h0 + sign * step * v
            values.append(loss())
        p.h0 = h0
        slope = (values[0] - values[1]) / (2 * step)
        assert abs(slope - float((p.dh0.double() * v.double()).sum())) <= 2e-3 * float(p.dh0.double().norm())


def test_reference_gradients_against_differences():
    """The reference itself, in 64 bits."""
    rng = np.random.default_rng(4)
    start, c = np.array([0, 0, 9, 20, 20]), 3
    x, z, dy = rng.standard_normal((3, 22, c))
    h0, dl = rng.standard_normal((2, 4, c))

    def loss(x, z, h0):
        y, last, _, _ = ref.forward(x, z, start, h0)
        return (y * dy).sum() + (last * dl).sum()
    y, _, off, _ = ref.forward(x, z, start, h0)
    grads, _ = ref.backward(x, z, y, off, start, h0, dy, dl)
    for k, v in enumerate((x, z, h0)):
        d = rng.standard_normal(v.shape)
        up, down = [a + (1e-5 * d if i == k else 0) for i, a in enumerate((x, z, h0))], \
                   [a - (1e-5 * d if i == k else 0) for i, a in enumerate((x, z, h0))]
        slope = (loss(*up) - loss(*down)) / 2e-5
        assert abs(slope - (grads[k] * d).sum()) <= 1e-8 * (1 + abs(slope))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("rows,channels,pad", [(1, 1, 0), (1, 2048, 0), (5, 33, 1), (64, 130, 8), (300, 8, 0)])
def test_single_tokens(kind, rows, channels, pad):
    p = Problem(rows, channels, [0, rows], kind, pad)
    rng = np.random.default_rng(rows)
    n_slots = rows + 9
    pool = torch.from_numpy(rng.standard_normal((n_slots + 1, channels)).astype(np.float32)).to(DEV)
    before = host(pool)
    slots = rng.permutation(n_slots)[:rows].astype(np.int32)
    if rows > 4:
        slots[1], slots[3] = -1, n_slots                    # no request: below and above the pool
    y = p.new(rows, channels + pad, dtype=TYPES[kind])
    zipml.scan_step(p.x, p.ld, p.z, p.ld, rows, channels, pool, n_slots, y, channels + pad,
                    slots=torch.from_numpy(slots).to(DEV))
    after = host(pool)
    live = (slots >= 0) & (slots < n_slots)
    touched = np.zeros(n_slots + 1, bool)
    touched[slots[live]] = True
    np.testing.assert_array_equal(after[~touched], before[~touched])
    x, z = host(p.x)[live], host(p.z)[live]
    start = np.arange(live.sum() + 1)
    want, _, off, _ = ref.forward(x, z, start, before[slots[live]])
    assert (np.abs(after[slots[live]] - want) <= off + 2.0 ** -23 * np.abs(want)).all()
    close(y[torch.from_numpy(live)][:, :channels], want, off, kind)
    assert (y[:, :channels][torch.from_numpy(~live)] == 0).all() and (y[:, channels:] == 9.0).all()


@pytest.mark.gpu
def test_prefill_then_single_tokens_is_one_sequence():
    """A prompt through the scan and its tail through single steps: the same states to fp32 rounding."""
    p = Problem(400, 96, [0, 400], "f32")
    whole = host(p.forward())
    q = Problem(400, 96, [0, 390], "f32")
    q.set(p.w.cpu())
    q.h0 = p.h0
    q.forward()
    h = q.last.clone()
    y = p.new(1, 96)
    _, _, off, _ = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
    for t in range(390, 400):
        zipml.scan_step(p.x[t], p.ld, p.z[t], p.ld, 1, 96, h, 1, y, 96)
        assert (np.abs(host(y)[0] - whole[t]) <= 2 * off[t] + 2.0 ** -22 * np.abs(whole[t])).all()


@pytest.mark.gpu
def test_same_bits_every_time():
    p = Problem(9000, 130, [0, 100, 8500, 9000], "f32")
    y = p.forward(train=True).clone()
    dx, dz = (v.clone() for v in p.backward())
    for _ in range(3):
        assert torch.equal(y, p.forward(train=True))
        bx, bz = p.backward()
        assert torch.equal(dx, bx) and torch.equal(dz, bz)


@pytest.mark.gpu
def test_in_a_graph():
    """Captured once, replayed with the program's own work in between, on new inputs each time."""
    p = Problem(1500, 72, [0, 700, 1500], "bf16")
    q = Problem(1500, 72, [0, 700, 1500], "bf16", seed=9)
    p.forward(train=True)
    p.backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    t, c = p.tokens, p.channels
    y, g = p.new(t, c, dtype=torch.bfloat16), p.new(t, p.ld, dtype=torch.bfloat16)
    with torch.cuda.graph(graph, stream=side):
        zipml.scan_forward(p.x, p.ld, p.z, p.ld, t, c, y, c, p.ws, seq_start=p.start_dev, n_seq=2, h0=p.h0, h_last=p.last,
                           act_x=p.ax, act_z=p.az, states=p.states, seed=5, epoch=3, tag=7)
        zipml.scan_backward(p.ax, p.az, p.states, p.dy, c, t, c, g, p.ld, g[:, p.zat:], p.ld, p.ws,
                            seq_start=p.start_dev, n_seq=2, h0=p.h0, dh_last=p.dh_last, dh0=p.dh0)
    both = [p.w.clone(), q.w.clone()]
    for k in range(4):
        p.w.copy_(both[k % 2])
        y.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), g[:, :c].clone(), g[:, p.zat:p.zat + c].clone()
        want = (p.forward(train=True), *p.backward())
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_sizes(lib):
    assert zipml.scan_workspace_bytes(1, 1) > 0
    assert zipml.scan_workspace_bytes(100000, 64) >= (100000 // 256) * 64 * 8
    for t, c in ((0, 1), (1, 0), (-1, 4), (1 << 41, 1), (1 << 40, 1 << 15), (1 << 31, 64)):
        assert zipml.scan_workspace_bytes(t, c) == 0


def test_refusals(lib):
    def fwd(x=FAKE, ldx=40, z=FAKE, ldz=40, dtype=zipml.BF16, t=10, c=40, seq=FAKE, n=2, h0=FAKE, y=FAKE, ldy=40,
            last=FAKE, ax=None, az=None, states=None, epoch=0, tag=0, ws=FAKE, nb=1 << 20):
        return lib.zipml_scan_forward(None, x, ldx, z, ldz, dtype, t, c, seq, n, h0, y, ldy, last, ax, az, states, 0, epoch,
                                      tag, ws, nb)
    for kw in ({"x": None}, {"z": None}, {"y": None}, {"ldx": 39}, {"ldz": 39}, {"ldy": 39}, {"dtype": 5}, {"t": 0}, {"c": 0},
               {"n": 0}, {"n": 1 << 31}, {"seq": None, "n": 2}, {"ax": FAKE}, {"ax": FAKE, "az": FAKE}, {"states": FAKE},
               {"epoch": 1 << 24}, {"tag": -1}, {"tag": 239}, {"ldx": 1 << 60}):
        assert fwd(**kw) == zipml.EINVAL, kw
    assert fwd(ws=None) == zipml.EWORKSPACE and fwd(nb=8) == zipml.EWORKSPACE
    for k in ("x", "z", "y", "seq", "h0", "last", "ws"):
        assert fwd(**{k: ODD}) == zipml.EALIGN, k
    assert fwd(ax=ODD, az=FAKE, states=FAKE) == zipml.EALIGN

    def bwd(ax=FAKE, az=FAKE, states=FAKE, dy=FAKE, ldy=40, dtype=zipml.F32, t=10, c=40, seq=FAKE, n=2, h0=FAKE, dl=FAKE,
            dx=FAKE, ldx=40, dz=FAKE, ldz=40, dh0=FAKE, ws=FAKE, nb=1 << 20):
        return lib.zipml_scan_backward(None, ax, az, states, dy, ldy, dtype, t, c, seq, n, h0, dl, dx, ldx, dz, ldz, dh0,
                                       ws, nb)
    for kw in ({"ax": None}, {"az": None}, {"states": None}, {"dy": None}, {"dx": None}, {"dz": None}, {"ldy": 39}, {"ldx": 39},
               {"ldz": 39}, {"dtype": -1}, {"t": 0}, {"c": -1}, {"n": 0}, {"seq": None, "n": 3}):
        assert bwd(**kw) == zipml.EINVAL, kw
    assert bwd(ws=None) == zipml.EWORKSPACE and bwd(nb=8) == zipml.EWORKSPACE
    for k in ("ax", "az", "states", "dy", "seq", "h0", "dl", "dx", "dz", "dh0", "ws"):
        assert bwd(**{k: ODD}) == zipml.EALIGN, k

    def step(x=FAKE, ldx=40, z=FAKE, ldz=40, dtype=zipml.F32, rows=4, c=40, h=FAKE, n=8, slots=FAKE, y=FAKE, ldy=40):
        return lib.zipml_scan_step(None, x, ldx, z, ldz, dtype, rows, c, h, n, slots, y, ldy)
    for kw in ({"x": None}, {"z": None}, {"h": None}, {"y": None}, {"ldx": 39}, {"ldz": 39}, {"ldy": 39}, {"dtype": 2},
               {"rows": 0}, {"c": 0}, {"n": 0}, {"slots": None, "n": 3}, {"rows": 1 << 32}):
        assert step(**kw) == zipml.EINVAL, kw
    for k in ("x", "z", "h", "slots", "y"):
        assert step(**{k: ODD}) == zipml.EALIGN, k


def test_mixed_types_are_refused(lib):
    a, b = torch.zeros(2), torch.zeros(2, dtype=torch.bfloat16)
    assert zipml._same_dtype(a, a, b) == -1 and zipml._same_dtype(b, b, b) == zipml.BF16
