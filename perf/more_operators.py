"""The operators of a layer whose product runs on 8-bit codes with a scale a row, as a user's program calls them.

  codes     rows are turned into 8-bit codes with one scale a row, and back: zipml.row8_encode, zipml.row8_decode
  norm      the residual is added, the sum normed by its root mean square, and the result comes out in codes:
            zipml.norm_forward (and zipml.row8_decode, which gives the values that the codes stand for)
  train     the same with its result in the inputs' type, then the backward pass: zipml.norm_forward,
            zipml.norm_backward
  product   a linear layer on codes of tokens and weights: zipml.row8_product
  clip      gradients of all layers scaled down to a largest norm, on their way into one bucket: zipml.clip

``run`` computes the same from elementary torch operations where ``own`` is false.

Codes are int8, rows a multiple of 16 bytes apart, zeros from the row's last value up to the next multiple of 16.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
STREAM = 16       # first Philox stream of stored values
LEAST = 2.0 ** -126
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------

def listed():
    return [
        # a gradient on its way into the backward product: fp32 rows of an odd width inside a wider tensor, unbiased rounding
        {"name": "codes odd fp32", "op": "codes", "rows": 1000, "cols": 1001, "pad": 3, "type": "f32", "draws": True},
        # a layer's input over a training batch
        {"name": "codes batch", "op": "codes", "rows": 16384, "cols": 4096, "pad": 0, "type": "bf16", "draws": False},
        # one request's token, the smallest call
        {"name": "norm one token", "op": "norm", "rows": 1, "cols": 2048, "pad": 0, "type": "bf16"},
        # a long prompt, or the forward half of a training step
        {"name": "norm batch", "op": "norm", "rows": 16384, "cols": 4096, "pad": 0, "type": "bf16"},
        # a small fp32 training step of odd sizes
        {"name": "norm train odd fp32", "op": "train", "rows": 1000, "cols": 1001, "pad": 3, "type": "f32"},
        # a training step over 16,384 tokens
        {"name": "norm train batch", "op": "train", "rows": 16384, "cols": 4096, "pad": 0, "type": "bf16"},
        # one request's token through a layer: the weights are read once
        {"name": "product one token", "op": "product", "rows": 1, "d_out": 4096, "d_in": 4096, "pad": 0, "type": "bf16",
         "bias": False},
        # 64 requests, few outputs and a long contraction
        {"name": "product requests", "op": "product", "rows": 64, "d_out": 1024, "d_in": 8192, "pad": 0, "type": "bf16",
         "bias": False},
        # a ragged batch through a layer of odd sizes, with a bias, to fp32
        {"name": "product odd fp32", "op": "product", "rows": 1000, "d_out": 1001, "d_in": 520, "pad": 16, "type": "f32",
         "bias": True},
        # a training batch
        {"name": "product large", "op": "product", "rows": 16384, "d_out": 4096, "d_in": 4096, "pad": 0, "type": "bf16",
         "bias": False},
        # one layer's gradients, of odd sizes
        {"name": "clip layer", "op": "clip", "layers": 1, "d": 1001, "channels": 520, "type": "f32", "out": "f32",
         "max_norm": 1.0},
        # the gradients of a whole model, fp32 as the weight gradient leaves them, into the bf16 bucket that is exchanged
        {"name": "clip model", "op": "clip", "layers": 24, "d": 2048, "channels": 2048, "type": "f32", "out": "bf16",
         "max_norm": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over the range: mostly 4, 5 or 7 times a power of two, as layers have them, sometimes any."""
    w = _log(rng, lo, hi)
    if rng.random() < 0.3 or w < 16:
        return w
    return (w >> w.bit_length() - 3 if (w >> w.bit_length() - 3) != 6 else 5) << w.bit_length() - 3


def draw(rng):
    op = rng.choice(["codes", "norm", "norm", "train", "train", "product", "product", "product", "product", "clip"])
    kind = rng.choice(["bf16", "bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 8, rng.randint(1, 63)])
    if op in ("codes", "norm", "train"):
        cols = _width(rng, 1, 16384)
        c = {"op": op, "rows": _log(rng, 1, max(1, min(65536, (1 << 25) // cols))), "cols": cols, "pad": pad, "type": kind}
        return {**c, "draws": rng.random() < 0.5} if op == "codes" else c
    if op == "product":
        d_out, d_in = _width(rng, 1, 16384), _width(rng, 1, 32768)
        most = min(65536, (1 << 37) // (d_out * d_in), (1 << 28) // d_in, (1 << 27) // d_out)
        return {"op": op, "rows": _log(rng, 1, max(1, most)), "d_out": d_out, "d_in": d_in, "pad": rng.choice([0, 0, 16, 48]),
                "type": kind, "bias": rng.random() < 0.3}
    d, channels = _width(rng, 8, 4096), _width(rng, 8, 4096)
    layers = _log(rng, 1, max(1, min(200, (1 << 27) // (3 * d * channels))))
    return {"op": op, "layers": layers, "d": d, "channels": channels, "type": kind, "out": rng.choice(["bf16", "f32"]),
            "max_norm": rng.choice([0.5, 1.0, 5.0, 1e6])}


# ---- inputs -----------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(g, rows, cols, pad, kind, size=1.0):
    """Roughly normal values whose scale differs by column, as activations have them, in rows of a wider tensor."""
    scale = torch.exp(0.7 * torch.randn(cols + pad, generator=g, device="cuda")) * size
    return (torch.randn(rows, cols + pad, generator=g, device="cuda") * scale).to(TYPES[kind])


def _wide(cols):
    return -(-cols // 16) * 16


def _codes(g, rows, cols, pad):
    """Codes and scales of rows of roughly normal values, rows pad bytes more apart than they need."""
    q = torch.zeros(rows, _wide(cols) + pad, dtype=torch.int8, device="cuda")
    q[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * 32.0).round_().clamp_(-127, 127).to(torch.int8)
    return q, torch.exp(0.5 * torch.randn(rows, generator=g, device="cuda")) * 0.02


def _sizes(case):
    """Values of each tensor of a model of so many layers: two projections and a gain each."""
    d, c = case["d"], case["channels"]
    return [2 * c * d, d * c, d] * case["layers"]


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    s = {"case": case, "seed": seed}
    if op == "clip":
        s["grads"] = [(torch.randn(n, generator=g, device="cuda") * 0.02).to(TYPES[case["type"]]) for n in _sizes(case)]
        return s
    if op == "product":
        s["x"], s["x_scales"] = _codes(g, case["rows"], case["d_in"], case["pad"])
        s["w"], s["w_scales"] = _codes(g, case["d_out"], case["d_in"], 0)
        s["bias"] = torch.randn(case["d_out"], generator=g, device="cuda") if case["bias"] else None
        return s
    rows, cols, pad, kind = case["rows"], case["cols"], case["pad"], case["type"]
    s["x"] = _activations(g, rows, cols, pad, kind)
    if op != "codes":
        s["add"] = _activations(g, rows, cols, pad, kind, 2.0)
        s["gain"] = 1.0 + 0.1 * torch.randn(cols, generator=g, device="cuda")
    if op == "train":
        s["dy"] = _activations(g, rows, cols, 0, kind, 0.02)
        s["dsum"] = _activations(g, rows, cols, 0, kind, 0.02)
    return s


# ---- the operators ----------------------------------------------------------------------------

def run(state):
    return _RUN[state["case"]["op"]](state)


_zipml = None


def _library():
    global _zipml
    if _zipml is None:
        from paper_1611_05402_amd import zipml
        _zipml = zipml
    return _zipml


def _new(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda")


def _codes_run(s):
    c, x = s["case"], s["x"]
    rows, cols = c["rows"], c["cols"]
    if not own:
        return _rounded(x[:, :cols].float(), s["seed"] if c["draws"] else None).to(torch.bfloat16)
    zipml = _library()
    if "out" not in s:                                     # what a program allocates once
        s.update(codes=_new(rows, _wide(cols), dtype=torch.int8), scales=_new(rows), out=_new(rows, cols, dtype=torch.bfloat16))
    zipml.row8_encode(x, rows, cols, x.stride(0), s["codes"], _wide(cols), s["scales"],
                      rounding=zipml.STOCHASTIC if c["draws"] else zipml.NEAREST, seed=s["seed"], epoch=0, tag=0)
    zipml.row8_decode(s["codes"], _wide(cols), s["scales"], rows, cols, s["out"], cols)
    return s["out"]


def _norm(s):
    c, x, add = s["case"], s["x"], s["add"]
    rows, cols = c["rows"], c["cols"]
    if not own:
        total, _, v = _normed(x[:, :cols], add[:, :cols], s["gain"])
        return {"sum": total, "y": _rounded(v, None).to(torch.bfloat16)}
    zipml = _library()
    if "out" not in s:
        s.update(total=_new(rows, cols, dtype=x.dtype), codes=_new(rows, _wide(cols), dtype=torch.int8), scales=_new(rows),
                 out=_new(rows, cols, dtype=torch.bfloat16))
    zipml.norm_forward(x, x.stride(0), rows, cols, EPS, gain=s["gain"], add=add, ldadd=add.stride(0), sum=s["total"], ldsum=cols,
                       codes=s["codes"], ldc=_wide(cols), scales=s["scales"])
    zipml.row8_decode(s["codes"], _wide(cols), s["scales"], rows, cols, s["out"], cols)
    return {"sum": s["total"], "y": s["out"]}


def _train(s):
    c, x, add, dy, dsum = s["case"], s["x"], s["add"], s["dy"], s["dsum"]
    rows, cols, kind = c["rows"], c["cols"], x.dtype
    if not own:
        total, rstd, v = _normed(x[:, :cols], add[:, :cols], s["gain"])
        n = total.float() * rstd
        a = dy.float() * s["gain"]
        dx = dsum.float() + rstd * (a - n * (a * n).mean(1, keepdim=True))
        return {"sum": total, "y": v.to(kind), "dx": dx.to(kind), "dgain": (dy.float() * n).sum(0)}
    zipml = _library()
    if "ws" not in s:
        s.update(total=_new(rows, cols, dtype=kind), y=_new(rows, cols, dtype=kind), dx=_new(rows, cols, dtype=kind),
                 rstd=_new(rows), dgain=_new(cols), ws=_new(zipml.norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8))
    zipml.norm_forward(x, x.stride(0), rows, cols, EPS, gain=s["gain"], add=add, ldadd=add.stride(0), sum=s["total"], ldsum=cols,
                       y=s["y"], ldy=cols, rstd=s["rstd"])
    zipml.norm_backward(dy, cols, s["total"], cols, rows, cols, s["rstd"], s["dx"], cols, s["ws"], gain=s["gain"], dsum=dsum,
                        lddsum=cols, dgain=s["dgain"])
    return {"sum": s["total"], "y": s["y"], "dx": s["dx"], "dgain": s["dgain"]}


def _product(s):
    c, x, w = s["case"], s["x"], s["w"]
    rows, d_out, d_in, kind = c["rows"], c["d_out"], c["d_in"], TYPES[c["type"]]
    if not own:
        y = x[:, :d_in].float() @ w[:, :d_in].float().t() * s["x_scales"].unsqueeze(1) * s["w_scales"]
        return (y if s["bias"] is None else y + s["bias"]).to(kind)
    zipml = _library()
    if "ws" not in s:
        s.update(y=_new(rows, d_out, dtype=kind),
                 ws=_new(zipml.row8_product_workspace_bytes(rows, d_out, d_in), dtype=torch.uint8))
    zipml.row8_product(x, x.stride(0), s["x_scales"], w, w.stride(0), s["w_scales"], rows, d_out, d_in, s["y"], d_out, s["ws"],
                       bias=s["bias"])
    return s["y"]


def _clip(s):
    c = s["case"]
    if not own:
        norm = torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt()
        factor = torch.where(norm <= c["max_norm"], 1.0, c["max_norm"] / norm).float()
        bucket = torch.cat([(t.float() * factor).to(TYPES[c["out"]]) for t in s["grads"]])
        return {"norm": norm.float(), "bucket": bucket}
    zipml = _library()
    if "ws" not in s:
        sizes = _sizes(c)
        s.update(bucket=_new(sum(sizes), dtype=TYPES[c["out"]]), norm=_new(2),
                 ws=_new(zipml.clip_workspace_bytes(len(sizes)), dtype=torch.uint8))
        s["list"] = zipml.ClipList(s["grads"], list(s["bucket"].split(sizes)))
    zipml.clip(s["list"], c["max_norm"], s["norm"], s["ws"])
    return {"norm": s["norm"][0], "bucket": s["bucket"]}


_RUN = {"codes": _codes_run, "norm": _norm, "train": _train, "product": _product, "clip": _clip}


# ---- plain form -------------------------------------------------------------------------------

def _philox(row, col8, stream, seed):
    """The four words of Philox4x32-10 for every (row, group of 8 columns)."""
    low = 0xFFFFFFFF
    c = [row & low, row >> 32, col8, torch.full_like(row, stream)]
    k = [seed & low, (seed >> 32) & low]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((q >> 32) & low) ^ c[1] ^ k[0], q & low, ((p >> 32) & low) ^ c[3] ^ k[1], p & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return c


def _rounded(v, seed):
    """What fp32 rows are after 8-bit codes with a scale a row: to the nearest code, or with a seed by its draws."""
    rows, cols = v.shape
    scale = (v.abs().amax(1, keepdim=True) / 127.0).clamp_min(LEAST)
    t = v * (1.0 / scale)
    if seed is None:
        return t.round() * scale
    wide = -(-cols // 8)
    row = torch.arange(rows, device=v.device).view(-1, 1).expand(rows, wide)
    col8 = torch.arange(wide, device=v.device).view(1, -1).expand(rows, wide)
    words = torch.stack(_philox(row, col8, STREAM, seed), -1)
    draws = torch.stack([words & 0xFFFF, words >> 16], -1).view(rows, wide * 8)[:, :cols]
    return torch.floor(t + (draws.float() + 0.5) / 65536.0).clamp(-127, 127) * scale


def _normed(x, add, gain):
    """(the sum in its type, 1 / root mean square, the normed values in fp32)."""
    total = (x.float() + add.float()).to(x.dtype)
    rstd = (1.0 / (total.double().square().mean(1, keepdim=True) + EPS).sqrt()).float()
    return total, rstd, total.float() * rstd * gain


# ---- the same from the definitions, in 64 bits ------------------------------------------------

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "clip":
        grads = [t.to(torch.float64) for t in s["grads"]]
        square = math.fsum(float(torch.dot(t, t)) for t in grads)
        norm = math.sqrt(square)
        by = 1.0 if norm <= case["max_norm"] else case["max_norm"] / norm
        return {"norm": norm, "bucket": torch.cat([t.mul_(by) for t in grads])}
    if op == "product":
        d_in = case["d_in"]
        x = s["x"][:, :d_in].to(torch.float64) * s["x_scales"].to(torch.float64)[:, None]
        w = s["w"][:, :d_in].to(torch.float64) * s["w_scales"].to(torch.float64)[:, None]
        y = torch.mm(x, w.t().contiguous())
        return y if s["bias"] is None else y.add_(s["bias"].to(torch.float64))
    cols = case["cols"]
    x = s["x"][:, :cols].to(torch.float64)
    if op == "codes":
        return _held(x, seed if case["draws"] else None)
    total = (x + s["add"][:, :cols].to(torch.float64)).to(s["x"].dtype).to(torch.float64)
    root = torch.sqrt((total ** 2).sum(1, keepdim=True) / cols + EPS)
    n, gain = total / root, s["gain"].to(torch.float64)
    if op == "norm":
        return {"sum": total, "y": _held(n * gain, None)}
    dy = s["dy"].to(torch.float64)
    a = dy * gain
    along = (a * n).sum(1, keepdim=True) / cols
    return {"sum": total, "y": n * gain, "dx": s["dsum"].to(torch.float64) + (a - along * n) / root,
            "dgain": (dy * n).sum(0)}


def _held(v, seed):
    """Codes times scales, by the published generator (Salmon et al., SC'11) where there is a seed."""
    rows, cols = v.shape
    step = torch.maximum(v.abs().max(1).values / 127.0, torch.tensor(LEAST, dtype=torch.float64, device=v.device))[:, None]
    if seed is None:
        return torch.round(v / step) * step
    units, mask = (cols + 7) // 8, (1 << 32) - 1
    words = [torch.arange(rows, device=v.device)[:, None].repeat(1, units), torch.zeros(rows, units, dtype=torch.int64, device=v.device),
             torch.arange(units, device=v.device)[None].repeat(rows, 1), torch.full((rows, units), STREAM, device=v.device)]
    key = [seed % (1 << 32), seed >> 32]
    for turn in range(10):
        first, second = words[0] * 0xD2511F53, words[2] * 0xCD9E8D57
        hi = [(w >> 16 >> 16) & mask for w in (first, second)]
        keys = [(key[0] + turn * 0x9E3779B9) & mask, (key[1] + turn * 0xBB67AE85) & mask]
        words = [hi[1] ^ words[1] ^ keys[0], second & mask, hi[0] ^ words[3] ^ keys[1], first & mask]
    halves = [h for w in words for h in (w % 65536, w // 65536)]
    draws = torch.stack(halves, 2).reshape(rows, units * 8)[:, :cols]
    return torch.floor(v / step + (draws.to(torch.float64) + 0.5) / 65536.0) * step


# ---- what one pass cannot do without ----------------------------------------------------------

def work(case):
    op, size = case["op"], 2 if case["type"] == "bf16" else 4
    if op == "clip":                                       # read once, written once
        n = sum(_sizes(case))
        return {"bytes": n * (size + (2 if case["out"] == "bf16" else 4)), "flops": 3 * n}
    if op == "product":
        rows, o, i = case["rows"], case["d_out"], case["d_in"]
        return {"bytes": (rows + o) * (i + 4) + rows * o * size + (4 * o if case["bias"] else 0), "flops": 2 * rows * o * i}
    n, rows = case["rows"] * case["cols"], case["rows"]
    if op == "codes":                                      # values in, codes and scales out and in, values out
        return {"bytes": n * (size + 2 + 2) + 8 * rows, "flops": 4 * n}
    if op == "norm":                                       # x and residual in, the sum out, codes out and in, values out
        return {"bytes": n * (3 * size + 2 + 2) + 8 * rows + 4 * case["cols"], "flops": 8 * n}
    # x, residual, dy and the sum's gradient in; the sum out and in; y and dx out
    return {"bytes": 8 * size * n + 8 * rows + 12 * case["cols"], "flops": 20 * n}
