"""A recurrent layer that trains on activations stored in 8 bits, and then serves single tokens.

    [x z] = U W_in^T,   y = scan(x, z),   out = y W_out^T

Nothing of the forward pass is kept in more than 8 bits a value for the backward pass: U and y (for the two weight
gradients) and x and z (for the recurrence's own) are stored by zipml, 33/32 of a byte each in place of two bytes.
The layer learns the map of a fixed one with other weights from documents of different lengths packed into one batch.

    python examples/recurrent_layer.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1611_05402_amd import zipml  # noqa: E402

DEV, BF16 = "cuda", torch.bfloat16


class RecurrentLayer:
    """Weights in fp32 with a bf16 copy for the products; buffers for batches of `tokens` tokens."""

    def __init__(self, d_in, channels, d_out, tokens, n_seq, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.d_in, self.c, self.d_out, self.tokens, self.n_seq = d_in, channels, d_out, tokens, n_seq
        self.w_in = torch.randn(2 * channels, d_in, generator=g, device=DEV) * d_in ** -0.5
        self.w_out = torch.randn(d_out, channels, generator=g, device=DEV) * channels ** -0.5
        self.seed, self.step_no = seed, 0
        new = lambda *s, dtype=BF16: torch.empty(*s, dtype=dtype, device=DEV)  # noqa: E731
        stored = lambda cols: new(zipml.act_bytes(tokens, cols), dtype=torch.uint8)  # noqa: E731
        self.act_u, self.act_x, self.act_z, self.act_y = stored(d_in), stored(channels), stored(channels), stored(channels)
        self.states = new(-(-tokens // zipml.SCAN_BLOCK), channels, dtype=torch.float32)
        self.y, self.dxz = new(tokens, channels), new(tokens, 2 * channels)
        self.last = new(n_seq, channels, dtype=torch.float32)
        self.dw_in, self.dw_out = torch.empty_like(self.w_in), torch.empty_like(self.w_out)
        self.ws = new(max(zipml.scan_workspace_bytes(tokens, channels),
                          zipml.act_wgrad_workspace_bytes(tokens, 2 * channels, d_in, BF16),
                          zipml.act_wgrad_workspace_bytes(tokens, d_out, channels, BF16)), dtype=torch.uint8)
        self.copy_weights()

    def copy_weights(self):
        self.b_in, self.b_out = self.w_in.to(BF16), self.w_out.to(BF16)

    def stored_bytes(self):
        return sum(t.numel() * t.element_size() for t in (self.act_u, self.act_x, self.act_z, self.act_y, self.states))

    def forward(self, u, start, train=True):
        """u: bf16 [tokens][d_in], documents back to back at the offsets `start`.  Returns out (bf16)."""
        t, c = self.tokens, self.c
        xz = u @ self.b_in.t()
        kw = {}
        if train:
            zipml.act_encode(u, t, self.d_in, u.stride(0), self.seed, self.step_no, 0, self.act_u)
            kw = dict(act_x=self.act_x, act_z=self.act_z, states=self.states, seed=self.seed, epoch=self.step_no, tag=1)
        zipml.scan_forward(xz[:, :c], 2 * c, xz[:, c:], 2 * c, t, c, self.y, c, self.ws, seq_start=start, n_seq=self.n_seq,
                           h_last=self.last, **kw)
        if train:
            zipml.act_encode(self.y, t, c, c, self.seed, self.step_no, 3, self.act_y)
        return self.y @ self.b_out.t()

    def backward(self, d_out, start):
        """Weight gradients in dw_in, dw_out from what the forward pass stored; returns the gradient of u."""
        t, c = self.tokens, self.c
        zipml.act_wgrad(d_out, self.d_out, self.act_y, t, self.d_out, c, self.dw_out, c, self.ws)
        dy = d_out @ self.b_out
        zipml.scan_backward(self.act_x, self.act_z, self.states, dy, c, t, c, self.dxz[:, :c], 2 * c, self.dxz[:, c:],
                            2 * c, self.ws, seq_start=start, n_seq=self.n_seq)
        zipml.act_wgrad(self.dxz, 2 * c, self.act_u, t, 2 * c, self.d_in, self.dw_in, self.d_in, self.ws)
        return self.dxz @ self.b_in

    def sgd(self, lr):
        self.w_in -= lr * self.dw_in
        self.w_out -= lr * self.dw_out
        self.copy_weights()
        self.step_no += 1

    def decode(self, u, pool, slots):
        """One token of each request: u bf16 [rows][d_in], states in rows `slots` (int32) of pool [n_slots][channels]."""
        rows, c = u.shape[0], self.c
        xz, y = u @ self.b_in.t(), torch.empty(u.shape[0], c, dtype=BF16, device=DEV)
        zipml.scan_step(xz[:, :c], 2 * c, xz[:, c:], 2 * c, rows, c, pool, pool.shape[0], y, c, slots=slots)
        return y @ self.b_out.t()


def documents(tokens, n_seq, seed):
    """Offsets of n_seq documents of different lengths that fill `tokens` tokens."""
    g = torch.Generator()
    g.manual_seed(seed)
    cut = torch.sort(torch.randint(0, tokens + 1, (n_seq - 1,), generator=g)).values
    return torch.cat([torch.tensor([0]), cut, torch.tensor([tokens])]).to(DEV)


def train(steps=60, tokens=4096, d_in=256, channels=512, d_out=256, n_seq=9, lr=0.2, say=print):
    """Returns the losses and the trained layer."""
    teacher = RecurrentLayer(d_in, channels, d_out, tokens, n_seq, seed=1)
    layer = RecurrentLayer(d_in, channels, d_out, tokens, n_seq, seed=2)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    losses = []
    for step in range(steps):
        u = torch.randn(tokens, d_in, generator=g, device=DEV).to(BF16)
        start = documents(tokens, n_seq, step)
        target = teacher.forward(u, start, train=False).float()
        out = layer.forward(u, start)
        diff = out.float() - target
        layer.backward((diff / tokens).to(BF16), start)
        layer.sgd(lr)
        losses.append((diff.square().sum() / (2 * tokens)).reshape(1))
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step:4d}  loss {losses[-1].item():.4f}")
    return torch.cat(losses).tolist(), layer


def serve(layer, say=print):
    """A prompt through the scan, its last tokens through single steps: returns the largest difference of the two ways."""
    t, n = layer.tokens, 16
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    u = torch.randn(t, layer.d_in, generator=g, device=DEV).to(BF16)
    starts = [torch.full((layer.n_seq + 1,), k, dtype=torch.int64, device=DEV) for k in (t, t - n)]
    for s in starts:
        s[0] = 0
    whole = layer.forward(u, starts[0], train=False)[-n:].float()
    layer.forward(u, starts[1], train=False)
    pool = torch.zeros(4, layer.c, device=DEV)
    slots = torch.tensor([2], dtype=torch.int32, device=DEV)
    pool[2] = layer.last[0]
    single = torch.cat([layer.decode(u[k:k + 1], pool, slots) for k in range(t - n, t)]).float()
    off = float((single - whole).abs().max() / whole.abs().max())
    say(f"{n} tokens one by one against all at once: largest difference {off:.1e} of the largest output")
    return off


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=60)
    a = p.parse_args()
    losses, layer = train(a.steps)
    held = layer.tokens * (layer.d_in + 3 * layer.c) * 2
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; kept for the backward pass: {layer.stored_bytes() / 2 ** 20:.2f} MiB "
          f"(bf16: {held / 2 ** 20:.2f} MiB)")
    serve(layer)


if __name__ == "__main__":
    main()
