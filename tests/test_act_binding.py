"""Tensors of a type or layout that the calls on stored activations would read as something else are refused by the binding before anything is
enqueued (no GPU needed): 32-bit offsets would be read to twice their length."""
import pytest
import torch

from paper_1611_05402_amd import zipml

BF16, F32 = torch.bfloat16, torch.float32
T, C, N = 8, 64, 2


class Went(Exception):
    """A call got as far as the library."""


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Went
        return call


@pytest.fixture(autouse=True)
def library(monkeypatch):
    monkeypatch.setattr(zipml, "lib", lambda L=Library(): L)
    monkeypatch.setattr(zipml, "_stream", lambda stream=None: None)
    monkeypatch.setattr(zipml, "strerror", lambda code: "refused")


def rows(dtype=BF16, apart=1):
    return torch.zeros(T, C * apart, dtype=dtype)[:, ::apart]


def act():
    return torch.zeros(T * (C + C // 32), dtype=torch.uint8)


def state(n=N, dtype=F32):
    return torch.zeros(n, C, dtype=dtype)


def forward(**kw):
    a = dict(x=rows(), z=rows(), y=rows(), seq_start=torch.tensor([0, 3, T]), h0=state(), h_last=state(), act_x=act(), act_z=act(),
             states=state(1))
    a.update(kw)
    x, z, y = a.pop("x"), a.pop("z"), a.pop("y")
    zipml.scan_forward(x, C, z, C, T, C, y, C, act(), n_seq=N, **a)


def backward(**kw):
    a = dict(act_x=act(), act_z=act(), states=state(1), dy=rows(), dx=rows(), dz=rows(), seq_start=torch.tensor([0, 3, T]), h0=state(),
             dh_last=state(), dh0=state())
    a.update(kw)
    ax, az, st, dy, dx, dz = (a.pop(k) for k in ("act_x", "act_z", "states", "dy", "dx", "dz"))
    zipml.scan_backward(ax, az, st, dy, C, T, C, dx, C, dz, C, act(), n_seq=N, **a)


def step(**kw):
    a = dict(x=rows(), z=rows(), h=state(T), y=rows(), slots=torch.arange(T, dtype=torch.int32))
    a.update(kw)
    zipml.scan_step(a["x"], C, a["z"], C, T, C, a["h"], T, a["y"], C, slots=a["slots"])


def wgrad(**kw):
    a = dict(dy=rows(), act=act(), dw=torch.zeros(C, C))
    a.update(kw)
    zipml.act_wgrad(a["dy"], C, a["act"], T, C, C, a["dw"], C, act())


def encode(**kw):
    zipml.act_encode(kw.get("x", rows()), T, C, C, 0, 0, 0, kw.get("act", act()))


def decode(**kw):
    zipml.act_decode(kw.get("act", act()), T, C, kw.get("out", rows()), C)


APART, OFFSETS = rows(apart=2), torch.tensor([0, 3, T])
GAPS, BYTES = torch.zeros(N, 2 * C)[:, ::2], torch.zeros(T, 2 * 99, dtype=torch.uint8)[:, :99]
WRONG = ([(forward, k, v) for k, v in
          [("x", APART), ("z", APART), ("y", APART), ("seq_start", OFFSETS.int()), ("seq_start", torch.zeros(6, dtype=torch.int64)[::2]),
           ("h0", state(dtype=BF16)), ("h0", state(dtype=torch.float64)), ("h0", GAPS), ("h_last", state(dtype=BF16)),
           ("h_last", GAPS), ("states", state(1, BF16)), ("act_x", BYTES), ("act_z", BYTES)]] +
         [(backward, k, v) for k, v in
          [("dy", APART), ("dx", APART), ("dz", APART), ("seq_start", OFFSETS.int()), ("h0", state(dtype=BF16)), ("dh_last", state(dtype=BF16)),
           ("dh_last", torch.zeros(1, C).expand(N, C)), ("dh0", state(dtype=BF16)), ("states", state(1, BF16)), ("act_x", BYTES)]] +
         [(step, k, v) for k, v in
          [("x", APART), ("z", APART), ("y", APART), ("h", state(T, BF16)), ("h", torch.zeros(T, 2 * C)[:, :C]),
           ("slots", torch.arange(T)), ("slots", torch.arange(2 * T, dtype=torch.int32)[::2])]] +
         [(wgrad, "dy", APART), (wgrad, "dw", torch.zeros(C, C, dtype=BF16)), (wgrad, "dw", torch.zeros(C, C).t()), (wgrad, "act", BYTES),
          (encode, "x", APART), (encode, "act", BYTES), (decode, "out", APART), (decode, "act", BYTES)])


@pytest.mark.parametrize("call,name,tensor", WRONG, ids=[f"{c.__name__}-{n}-{i}" for i, (c, n, _) in enumerate(WRONG)])
def test_refused(call, name, tensor):
    with pytest.raises(zipml.ZipmlError) as e:
        call(**{name: tensor})
    assert e.value.code == zipml.EINVAL


@pytest.mark.parametrize("call", [forward, backward, step, wgrad, encode, decode])
def test_what_is_right_goes_on(call):
    with pytest.raises(Went):
        call()


def test_rows_of_one_value_may_lie_anyhow():
    assert zipml._rows("here", torch.zeros(T, 2)[:, :1], torch.zeros(1, T).t(), torch.zeros(())) == zipml.F32


def test_types_that_differ_are_refused_by_the_library():
    assert zipml._rows("here", rows(), rows(), rows(F32)) == zipml._rows("here", rows(torch.float16)) == -1
    assert zipml._rows("here", rows(), rows(F32), rows(apart=1)) == -1 and zipml._rows("here", rows(), rows(), rows()) == zipml.BF16


@pytest.mark.parametrize("call,name", [(wgrad, "dy"), (wgrad, "dw"), (wgrad, "act"), (encode, "x"), (encode, "act"), (decode, "out"), (decode, "act"),
                                       (step, "h"), (step, "slots")])
def test_none_is_for_the_library_to_refuse(call, name):
    with pytest.raises(Went):
        call(**{name: None})
