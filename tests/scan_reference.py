"""The gated recurrence from its definition, token by token in 64 bits (numpy), with bounds on what fp32 may be off.

A gate computed in fp32 is within (6 + 2 |z|) * 2^-24 of itself: |z| * 2^-24 * log2(e) from the argument of the power,
a few units in the last place from the power, the sum, the reciprocal and the product.  `eps` is that bound; it
also covers the two roundings of a step f h + g x.  The bounds follow the recurrences themselves.
A state keeps at least 2^-126 of what a run of tokens hands on, which is far below them."""
import numpy as np

BLOCK = 256


def sigmoid(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


def eps(z):
    return (6.0 + 2.0 * np.abs(z)) * 2.0 ** -24


def forward(x, z, start, h0):
    """(y, h_last, bound on y): x, z [tokens][channels], start [n + 1], h0 [n][channels]."""
    f, g = sigmoid(z), sigmoid(-z)
    e = eps(np.clip(z, -60, 60))
    y, off, last = np.zeros_like(x), np.zeros_like(x), h0.copy()
    last_off = np.zeros_like(h0)
    for s in range(len(start) - 1):
        h, o = h0[s], np.zeros_like(h0[s])
        for t in range(start[s], start[s + 1]):
            o = f[t] * o + e[t] * (2 * np.abs(f[t] * h) + 2 * np.abs(g[t] * x[t]))
            h = f[t] * h + g[t] * x[t]
            y[t], off[t] = h, o
        last[s], last_off[s] = h, o
    return y, last, off, last_off


def backward(x, z, y, y_off, start, h0, dy, dh_last):
    """Gradients from the stored x, z; y: the forward pass's exact states.  Returns (dx, dz, dh0) and their bounds."""
    f, g = sigmoid(z), sigmoid(-z)
    e = eps(z)
    dx, dz, dh0 = np.zeros_like(x), np.zeros_like(x), dh_last.copy()
    ox, oz, oh = np.zeros_like(x), np.zeros_like(x), np.zeros_like(dh_last)
    for s in range(len(start) - 1):
        a, b = start[s], start[s + 1]
        before, off = np.zeros((b - a,) + x.shape[1:]), np.zeros((b - a,) + x.shape[1:])
        h, o = h0[s], np.zeros_like(h0[s])
        for t in range(a, b):
            if t % BLOCK == 0 and t > a:
                h, o = y[t - 1], y_off[t - 1]
            before[t - a], off[t - a] = h, o
            o = f[t] * o + e[t] * (2 * np.abs(f[t] * h) + 2 * np.abs(g[t] * x[t]))
            h = f[t] * h + g[t] * x[t]
        right, o = dh_last[s], np.zeros_like(dh_last[s])
        for t in range(b - 1, a - 1, -1):
            d = dy[t] + right
            o = o + 2.0 ** -23 * (np.abs(dy[t]) + np.abs(right))
            w = before[t - a] - x[t]
            dx[t], ox[t] = g[t] * d, g[t] * o + 2 * e[t] * np.abs(g[t] * d)
            dz[t] = d * w * f[t] * g[t]
            oz[t] = f[t] * g[t] * (o * np.abs(w) + np.abs(d) * (off[t - a] + 4 * e[t] * (np.abs(before[t - a]) + np.abs(x[t]))))
            right, o = f[t] * d, f[t] * o + 2 * e[t] * np.abs(f[t] * d)
        dh0[s], oh[s] = right, o
    return (dx, dz, dh0), (ox, oz, oh)
