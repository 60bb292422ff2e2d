"""Gates that are nearly open (z of 8 to 17): what a state forgets at a token is then a fraction g = 1 - f of it that fp32 cannot see in f, so an
f that is off by its last bit is off in the same direction at every token.  Held against 64 bits in units of the state.

u = 2^-24, S the largest state of a channel.  What is allowed after n tokens:
  the gate     g is within eg = (6 + 2 |z|) u of itself, and takes the state that part nearer to x at every token: 2 eg S in all;
  the sums     what a block of 256 tokens forgets and what it adds are sums of positive terms over 8 tokens, 4 to 8 runs
               and 8 waves, each term a few products: within 32 u of themselves each, which moves a state by 64 u S at most;
  a block      the state within a block comes through at most 8 tokens (f within 4 u, a rounding), 32 runs (A within 2 u, a rounding) and
               8 waves (the same): 160 u S, not carried on;
  the chain    for each 32 blocks (8,192 tokens) the A of each block is rounded once (u / 2, A being above 1/2), 24 products of them once,
               the state nine times (u): 37 u S.
"""
import numpy as np
import pytest
import torch

import scan_reference as ref
from paper_1611_05402_amd import zipml

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24
GATES = np.array([4.0, 8.0, 10.0, 12.0, 14.0, 15.0, 16.0, 17.0])


def allowed(z, tokens):
    return (2 * (6 + 2 * np.abs(z)) + 64 + 160 + 37 * -(-tokens // 8192)) * U


def run(x, z, h0, train=False):
    """(y, h_last, what the backward pass needs) of one sequence, fp32."""
    tokens, c = x.shape
    y, last = torch.empty(tokens, c, device=DEV), torch.empty(1, c, device=DEV)
    ws = torch.empty(zipml.scan_workspace_bytes(tokens, c), dtype=torch.uint8, device=DEV)
    kept = {}
    if train:
        kept = dict(act_x=torch.empty(zipml.act_bytes(tokens, c), dtype=torch.uint8, device=DEV),
                    act_z=torch.empty(zipml.act_bytes(tokens, c), dtype=torch.uint8, device=DEV),
                    states=torch.empty(-(-tokens // zipml.SCAN_BLOCK), c, device=DEV))
    zipml.scan_forward(x, c, z, c, tokens, c, y, c, ws, h0=h0, h_last=last, **kept)
    return y, last, kept, ws


@pytest.mark.parametrize("copies", [1, 5])                  # workgroups of 32 channels and of 64
@pytest.mark.parametrize("tokens", [3000, 131072])
def test_constant_gates(tokens, copies):
    """x = 1 from the states 0, 1 and 3: h = 1 + (h0 - 1) f^t in closed form."""
    z, h0 = (np.tile(v.reshape(-1), copies) for v in np.meshgrid(GATES, [0.0, 1.0, 3.0]))
    c = z.size
    y, last, _, _ = run(torch.ones(tokens, c, device=DEV), torch.tensor(z, dtype=torch.float32, device=DEV).expand(tokens, c).contiguous(),
                        torch.tensor(h0, dtype=torch.float32, device=DEV).view(1, c))
    t = np.arange(1, tokens + 1)[:, None]
    want = 1 + (h0 - 1) * np.exp(-np.log1p(np.exp(-z)) * t)
    off = np.abs(y.double().cpu().numpy() - want) / np.maximum(h0, 1)
    assert (off <= allowed(z, tokens)).all(), off.max(0) / allowed(z, tokens)
    assert torch.equal(last[0], y[-1])


def test_gates_and_inputs_that_vary():
    tokens, c = 60000, 40
    rng = np.random.default_rng(5)
    x, z = (torch.from_numpy(v.astype(np.float32)).to(DEV) for v in (rng.standard_normal((tokens, c)) + 0.5,
                                                                     rng.uniform(9, 17, (tokens, c))))
    h0 = torch.from_numpy(rng.standard_normal((1, c)).astype(np.float32)).to(DEV)
    y, _, _, _ = run(x, z, h0)
    xs, f, g, h = x.double().cpu().numpy(), ref.sigmoid(z.double().cpu().numpy()), ref.sigmoid(-z.double().cpu().numpy()), h0.double().cpu().numpy()[0]
    want = np.zeros_like(xs)
    for t in range(tokens):
        h = f[t] * h + g[t] * xs[t]
        want[t] = h
    top = np.maximum(np.abs(xs).max(0), np.abs(want).max(0))
    assert (np.abs(y.double().cpu().numpy() - want) <= allowed(17.0, tokens) * top).all()


@pytest.mark.parametrize("copies", [1, 5])
@pytest.mark.parametrize("tokens", [3000, 131072])
@pytest.mark.parametrize("every", [0.0, 1.0])
def test_gradients_through_constant_gates(tokens, copies, every):
    """dy = `every` at all tokens and 1 (dh_last) at the last: d_t = every (1 - f^n) / g + f^(n - 1), n tokens from t on; dx = g d, dh0 = f d.  The
    stored gates are those of the forward pass exactly (quarters, the largest of a group 16)."""
    z = np.tile(np.append(GATES[:-1], [16.0] * 25), copies)     # groups of 32 channels
    c = z.size
    zt = torch.tensor(z, dtype=torch.float32, device=DEV).expand(tokens, c).contiguous()
    _, _, kept, ws = run(torch.ones(tokens, c, device=DEV), zt, None, train=True)
    dy = torch.full((tokens, c), every, device=DEV)
    dx, dz, dh0 = torch.empty(tokens, c, device=DEV), torch.empty(tokens, c, device=DEV), torch.empty(1, c, device=DEV)
    zipml.scan_backward(kept["act_x"], kept["act_z"], kept["states"], dy, c, tokens, c, dx, c, dz, c, ws,
                        dh_last=torch.ones(1, c, device=DEV), dh0=dh0)
    g, rate = 1 / (1 + np.exp(z)), np.log1p(np.exp(-z))
    n = np.arange(tokens, 0, -1)[:, None]
    d = every * -np.expm1(-rate * n) / g + np.exp(-rate * (n - 1))
    top = d.max(0)
    # (a product with g more)
    assert (np.abs(dx.double().cpu().numpy() - g * d) <= g * top * (allowed(z, tokens) + (8 + 2 * z) * U)).all()
    assert (np.abs(dh0.double().cpu().numpy()[0] - d[0] / (1 + np.exp(-z))) <= top * (allowed(z, tokens) + 4 * U)).all()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_single_tokens_hold_a_state_that_equals_its_input(kind):
    """h = x is where the recurrence stays: with an open gate b - g h is what one rounding of b leaves, below half an ulp of h, so
    the state moves by nothing; with a shut one f + g is within 4 u of 1 and what is off does not add up beyond 1 / g < 2 tokens."""
    z = torch.tensor([-9.0, -1.0, 0.0, 1.0, *GATES, float("inf")], dtype=kind, device=DEV).view(1, -1)
    c = z.shape[1]
    x = torch.full((1, c), 1.375, dtype=kind, device=DEV)
    pool, y = torch.full((1, c), 1.375, device=DEV), torch.empty(1, c, dtype=kind, device=DEV)
    for _ in range(3000):
        zipml.scan_step(x, c, z, c, 1, c, pool, 1, y, c)
    assert ((pool.double() - 1.375).abs() <= 16 * U * 1.375).all(), pool


@pytest.mark.parametrize("z", [3.0, 12.0])
def test_an_infinity_stays_one(z):
    """Through half-open and open gates, many tokens at once and one by one: f times an infinity is one."""
    tokens, c = 20000, 33
    x = torch.ones(tokens, c, device=DEV)
    x[300, 4], x[9000, 32] = float("inf"), float("-inf")
    y, last, _, _ = run(x, torch.full((tokens, c), z, device=DEV), None)
    assert (y[300:, 4] == float("inf")).all() and (y[9000:, 32] == float("-inf")).all()
    y[300:, 4] = y[9000:, 32] = 0
    assert torch.isfinite(y).all()
    out = torch.empty(1, c, device=DEV)
    zipml.scan_step(x[:1], c, torch.full((1, c), z, device=DEV), c, 1, c, last, 1, out, c)
    assert out[0, 4] == float("inf") and out[0, 32] == float("-inf") and torch.equal(out, last)
