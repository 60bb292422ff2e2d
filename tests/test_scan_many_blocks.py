"""The recurrence at sizes of more than 128 blocks of 256 tokens x 64 channels, where a workgroup takes 64 channels
and not 32; definitions and error bounds are those of test_scan."""
import numpy as np
import pytest
import torch

import act_reference as act
import scan_reference as ref
from paper_1611_05402_amd import zipml
from test_scan import Problem, TYPES, close, host
from test_scan import test_forward as forward_is_right
from test_scan import test_training_step as training_step_is_right

pytestmark = pytest.mark.gpu
KINDS = pytest.mark.parametrize("kind", ["bf16", "f32"])
SHAPES = [(1, 8257, "one"), (255, 8257, "empty ones"), (300, 4165, "single tokens"), (300, 4200, "nowhere"), (257, 4164, "no token"),
          (2570, 777, "filled up"), (2570, 780, "one"), (33500, 2, "empty ones"), (9001, 256, "empty ones")]


@KINDS
@pytest.mark.parametrize("tokens,channels,seqs", SHAPES)
def test_training_step(kind, tokens, channels, seqs):
    training_step_is_right(kind, tokens, channels, seqs)


@KINDS
@pytest.mark.parametrize("tokens,channels,seqs", SHAPES[-3:])
def test_forward(kind, tokens, channels, seqs):
    forward_is_right(kind, tokens, channels, seqs)


@KINDS
def test_on_either_side_of_the_limit(kind):
    """The same sequences with 128 blocks and, more channels beside them, with 136: the shared channels agree to rounding."""
    got = []
    for channels in (1024, 1088):
        p = Problem(2048, 1088, [0, 700, 2048], kind)
        p.channels, p.x, p.z = channels, p.x[:, :channels], p.z[:, :channels]
        p.h0, p.dh_last = p.h0[:, :channels].contiguous(), p.dh_last[:, :channels].contiguous()
        p.dy = p.dy[:, :channels].contiguous()
        p.ws = torch.empty(zipml.scan_workspace_bytes(2048, channels), dtype=torch.uint8, device="cuda")
        y = p.forward(train=True)
        want, _, off, _ = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
        close(y, want, off, kind)
        got.append((host(y)[:, :1024], 2 * off[:, :1024] + 2.0 ** -7 * np.abs(want[:, :1024]) * (kind == "bf16")))
    assert (np.abs(got[0][0] - got[1][0]) <= got[0][1] + 1e-30).all()


@KINDS
def test_gates_that_are_saturated(kind):
    c = 1100
    p = Problem(2000, c, [0, 2000], kind)
    w = p.w.cpu()
    big = torch.finfo(TYPES[kind]).max
    for k, v in enumerate([float("inf"), float("-inf"), big, -big, 40.0, -40.0, 17.0, -17.0]):
        w[:, p.zat + 137 * k] = v
        w[k::11, p.zat + 3] = v
    p.set(w)
    y = p.forward(train=True)
    want, _, off, _ = ref.forward(host(p.x), host(p.z), p.start, p.h0_host())
    close(y, want, off, kind)
    dx, dz = p.backward()
    qx = act.decode(*act.encode(p.x.float().cpu().numpy(), 5, 3, 7), c)
    qz = act.decode(*act.encode(np.clip(p.z.float().cpu().numpy(), -16, 16), 5, 3, 8), c)
    g, o = ref.backward(qx, qz, want, off, p.start, p.h0_host(), host(p.dy), host(p.dh_last))
    close(dx, g[0], o[0], kind)
    close(dz, g[1], o[1], kind)


@KINDS
def test_nan_and_infinity_stay_in_their_sequence(kind):
    tokens, c, start = 2000, 1100, [3, 900, 900, 1500, 1990]
    p = Problem(tokens, c, start, kind, scale_z=0.1, mean_z=0.0)               # f near 1/2
    clean = host(p.forward())
    w = p.w.cpu()
    w[100, 5] = float("nan")
    w[200, p.zat + 1040] = float("nan")
    w[0:3] = float("nan")
    w[1990:] = float("inf")
    p.set(w)
    y = host(p.forward(train=True))
    bad = np.zeros_like(clean, bool)
    bad[100:900, 5] = bad[200:900, 1040] = True
    assert np.isnan(y[bad]).all()
    np.testing.assert_array_equal(y[~bad], clean[~bad])
    dx, dz = (host(v) for v in p.backward())
    for v in (dx, dz):
        assert np.isfinite(v[900:]).all() and (v[:3] == 0).all() and (v[1990:] == 0).all()
    assert np.isfinite(host(p.dh0)[1:]).all() and np.isnan(dz[101:900, 5]).all()


def test_more_blocks_than_start_together():
    forward_is_right("bf16", 270000, 5, "empty ones")


def test_same_bits_every_time_and_in_a_graph():
    """Captured once, replayed with the program's own work in between; every replay and every eager pass gives the same bits."""
    p = Problem(9000, 290, [0, 100, 8500, 9000], "bf16")
    y, (dx, dz) = p.forward(train=True).clone(), (v.clone() for v in p.backward())
    t, c = p.tokens, p.channels
    out, g = p.new(t, c, dtype=torch.bfloat16), p.new(t, p.ld, dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        zipml.scan_forward(p.x, p.ld, p.z, p.ld, t, c, out, c, p.ws, seq_start=p.start_dev, n_seq=3, h0=p.h0, h_last=p.last,
                           act_x=p.ax, act_z=p.az, states=p.states, seed=5, epoch=3, tag=7)
        zipml.scan_backward(p.ax, p.az, p.states, p.dy, c, t, c, g, p.ld, g[:, p.zat:], p.ld, p.ws,
                            seq_start=p.start_dev, n_seq=3, h0=p.h0, dh_last=p.dh_last, dh0=p.dh0)
    for _ in range(4):
        out.fill_(3.0)
        g.fill_(3.0)
        p.ws.fill_(0xAB)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, y) and torch.equal(g[:, :c], dx) and torch.equal(g[:, p.zat:p.zat + c], dz)
        assert torch.equal(p.forward(train=True), y)
        ex, ez = p.backward()
        assert torch.equal(ex, dx) and torch.equal(ez, dz)
