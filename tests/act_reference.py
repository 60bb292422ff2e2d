"""Activations stored in 8 bits, from the definition, in 64 bits (numpy; shares no code with the library)."""
import numpy as np

U = np.uint64
LOW = U(0xFFFFFFFF)


def philox(row, col8, stream, seed, epoch):
    c = [row & LOW, row >> U(32), col8.astype(U), np.full_like(row, (epoch << 8) | stream)]
    k = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
    for _ in range(10):
        p, q = c[0] * U(0xD2511F53), c[2] * U(0xCD9E8D57)
        c = [(q >> U(32)) ^ c[1] ^ U(k[0]), q & LOW, (p >> U(32)) ^ c[3] ^ U(k[1]), p & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def draws(rows, wide, seed, epoch, tag, row0=0):
    """The 16-bit draw of every value of `rows` rows of a tensor from row0 on (wide, its width, a multiple of 8)."""
    row = np.repeat(np.arange(row0, row0 + rows, dtype=U), wide // 8)
    col8 = np.tile(np.arange(wide // 8, dtype=U), rows)
    w = np.stack(philox(row, col8, 16 + tag, seed, epoch), -1)
    return np.stack([w & U(0xFFFF), w >> U(16)], -1).reshape(rows, wide).astype(np.int64)


def encode(x, seed=0, epoch=0, tag=0, row0=0):
    """(codes int8 [rows][padded], exponent bytes uint8 [rows][padded / 32]) of fp32 values x, rows of a tensor from row0 on."""
    rows, cols = x.shape
    wide = -(-cols // 32) * 32
    v = np.zeros((rows, wide))
    v[:, :cols] = x
    g = v.reshape(rows, wide // 32, 32)
    bad = ~np.isfinite(g).all(-1)
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(g), g, 0.0)).max(-1))
    mant, exp = np.frexp(top)                              # top = mant * 2^exp, mant in [0.5, 1)
    e = np.where(top > 0, exp - 7 + (mant > 127.0 / 128.0), -126)
    e = np.maximum(e, -126)
    step = np.exp2(e.astype(float))[..., None]
    k = draws(rows, wide, seed, epoch, tag, row0).reshape(g.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        # the sum is rounded to fp32, as the definition has it
        t = ((g / step).astype(np.float32) + ((k + 0.5) / 65536.0).astype(np.float32)).astype(np.float32)
        codes = np.where(bad[..., None], 0.0, np.floor(t))
    return codes.astype(np.int8).reshape(rows, wide), np.where(bad, 255, e + 127).astype(np.uint8)


def decode(codes, byte, cols):
    rows, wide = codes.shape
    step = np.exp2(byte.astype(float) - 127.0)
    step[byte == 255] = np.nan
    step[byte == 0] = 0.0
    return (codes.reshape(rows, wide // 32, 32) * step[..., None]).reshape(rows, wide)[:, :cols]


def pack(codes, byte):
    """One buffer, as the library lays it out."""
    return np.concatenate([codes.view(np.uint8).reshape(-1), byte.reshape(-1)])
