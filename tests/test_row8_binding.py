"""Tensors of a type, layout or place that the calls on rows of codes, the norm and clipping would read as something else are refused by the
binding before anything is enqueued (no GPU needed)."""
import pytest
import torch

from paper_1611_05402_amd import zipml

BF16, F32 = torch.bfloat16, torch.float32
T, C, O = 6, 48, 5


class Went(Exception):
    """A call got as far as the library."""


class Library:
    def __getattr__(self, name):
        def call(*args):
            self.args = args
            raise Went
        return call


@pytest.fixture(autouse=True)
def library(monkeypatch):
    monkeypatch.setattr(zipml, "lib", lambda L=Library(): L)
    monkeypatch.setattr(zipml, "_stream", lambda stream=None: None)
    monkeypatch.setattr(zipml, "_here", lambda: -1)        # where CPU tensors are
    monkeypatch.setattr(zipml, "strerror", lambda code: "refused")


def rows(dtype=BF16, n=T, cols=C, apart=1):
    return torch.zeros(n, cols * apart, dtype=dtype)[:, ::apart]


def codes(n=T, **kw):
    return rows(torch.int8, n, **kw)


def floats(n):
    return torch.zeros(n)


def encode(**kw):
    a = dict(x=rows(), codes=codes(), scales=floats(T))
    a.update(kw)
    zipml.row8_encode(a["x"], T, C, C, a["codes"], C, a["scales"])


def decode(**kw):
    a = dict(codes=codes(), scales=floats(T), out=rows())
    a.update(kw)
    zipml.row8_decode(a["codes"], C, a["scales"], T, C, a["out"], C)


def product(**kw):
    a = dict(x=codes(), x_scales=floats(T), w=codes(O), w_scales=floats(O), bias=floats(O), y=rows(cols=O), workspace=floats(64))
    a.update(kw)
    zipml.row8_product(a["x"], C, a["x_scales"], a["w"], C, a["w_scales"], T, O, C, a["y"], O, a["workspace"], bias=a["bias"])


def forward(**kw):
    a = dict(gain=floats(C), add=rows(), sum=rows(), y=rows(), codes=codes(), scales=floats(T), rstd=floats(T))
    a.update(kw)
    zipml.norm_forward(a.pop("x", rows()), C, T, C, 1e-6, ldadd=C, ldsum=C, ldy=C, ldc=C, **a)


def backward(**kw):
    a = dict(dy=rows(), sum=rows(), rstd=floats(T), dx=rows(), workspace=floats(64), gain=floats(C), dsum=rows(), dgain=floats(C))
    a.update(kw)
    zipml.norm_backward(a["dy"], C, a["sum"], C, T, C, a["rstd"], a["dx"], C, a["workspace"], gain=a["gain"], dsum=a["dsum"], lddsum=C,
                        dgain=a["dgain"])


def clip(**kw):
    a = dict(grads=[floats(8), rows()], norm=floats(2), workspace=floats(4096))
    a.update(kw)
    zipml.clip(zipml.ClipList(a["grads"], a.get("outs")), 1.0, a["norm"], a["workspace"])


APART, GAPS = rows(apart=2), torch.zeros(2 * C)[::2]
WRONG = ([(encode, k, v) for k, v in [("x", APART), ("codes", codes(apart=2)), ("codes", codes().view(torch.uint8)), ("codes", rows()),
                                       ("scales", floats(T).double()), ("scales", rows(F32, T, 2)[:, 0])]] +
         [(decode, k, v) for k, v in [("out", APART), ("codes", codes(apart=2)), ("codes", rows()), ("scales", floats(T).to(BF16))]] +
         [(product, k, v) for k, v in [("x", codes(apart=2)), ("x", rows()), ("w", codes(O, apart=2)), ("w", rows(n=O)), ("y", rows(cols=O, apart=2)),
                                        ("x_scales", floats(T).to(BF16)), ("w_scales", torch.zeros(2 * O)[::2]), ("bias", floats(O).to(BF16))]] +
         [(forward, k, v) for k, v in [("x", APART), ("add", APART), ("add", rows(F32)), ("sum", rows(F32)), ("sum", APART), ("y", rows(F32)),
                                        ("y", APART), ("gain", floats(C).to(BF16)), ("gain", GAPS), ("codes", rows()), ("codes", codes(apart=2)),
                                        ("scales", floats(T).double()), ("rstd", floats(T).to(BF16))]] +
         [(backward, k, v) for k, v in [("dy", APART), ("sum", rows(F32)), ("dsum", rows(F32)), ("dsum", APART), ("dx", rows(F32)), ("dx", APART),
                                         ("rstd", floats(T).to(BF16)), ("gain", GAPS), ("dgain", floats(C).to(BF16)), ("dgain", GAPS)]] +
         [(clip, "norm", floats(1)), (clip, "norm", floats(2).to(BF16)), (clip, "grads", [rows(apart=2)]), (clip, "grads", [floats(4).double()])])


@pytest.mark.parametrize("call,name,tensor", WRONG, ids=[f"{c.__name__}-{n}-{i}" for i, (c, n, _) in enumerate(WRONG)])
def test_refused(call, name, tensor):
    with pytest.raises(zipml.ZipmlError) as e:
        call(**{name: tensor})
    assert e.value.code == zipml.EINVAL


CALLS = [encode, decode, product, forward, backward, clip]


@pytest.mark.parametrize("call", CALLS)
def test_what_is_right_goes_on(call):
    with pytest.raises(Went):
        call()


@pytest.mark.parametrize("call", CALLS)
def test_another_device_is_refused(call, monkeypatch):
    """A kernel may not reach another device's memory (nor the host's)."""
    monkeypatch.setattr(zipml, "_here", lambda: 0)
    with pytest.raises(zipml.ZipmlError) as e:
        call()
    assert e.value.code == zipml.EINVAL


@pytest.mark.parametrize("call,name", [(encode, "codes"), (encode, "scales"), (decode, "scales"), (product, "x"), (product, "workspace"),
                                       (product, "bias"), (forward, "y"), (forward, "gain"), (backward, "sum"), (backward, "workspace"),
                                       (clip, "norm"), (clip, "workspace")])
def test_none_is_for_the_library_to_judge(call, name):
    with pytest.raises(Went):
        call(**{name: None})


def test_types_the_library_does_not_have():
    for call, name in ((encode, "x"), (decode, "out"), (product, "y")):
        with pytest.raises(Went):
            call(**{name: rows(torch.float16, cols=O if call is product else C)})
        assert -1 in zipml.lib().args


def test_rows_of_one_value_may_lie_anyhow():
    assert zipml._row("here", "x", torch.zeros(T, 2)[:, :1], F32, -1) and zipml._row("here", "x", torch.zeros(1, T).t(), F32, -1)
