"""Microscaled 4-bit floats and the operators on them, in 64 bits, from their definitions."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
BLOCK = 32


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def scales(v):
    """The scale byte of every block of rows (R, C)."""
    R, C = v.shape
    b = np.zeros((R, blocks(C) * BLOCK))
    b[:, :C] = v
    m = np.abs(b).reshape(R, -1, BLOCK).max(2) if C else np.zeros((R, 0))
    s = np.full(m.shape, -127.0)
    some = np.isfinite(m) & (m > 0)
    # the least s with m < 7 * 2^s (m / 7 is never a power of two: 7 * 2^s is, in 64 bits, its own border)
    guess = np.floor(np.log2(m[some] / 7))
    for step in (-1, 0, 1, 2):
        fits = (m[some] < 7 * 2.0 ** (guess + step)) & ~(m[some] < 7 * 2.0 ** (guess + step - 1))
        s[some] = np.where(fits, np.maximum(guess + step, -127), s[some])
    return np.where(np.isfinite(m), s + 127, 255).astype(np.uint8)


def codes(v, scale):
    """Codes (R, C), 0 to 15, of rows under the scales of their blocks: the nearest value, ties to the even code."""
    R, C = v.shape
    b = np.repeat(scale.astype(float), BLOCK, 1)[:, :C]
    with np.errstate(invalid="ignore", over="ignore"):
        q = np.abs(v) * 2.0 ** (127 - b)
        d = np.abs(np.minimum(q, 6)[..., None] - VALUES)
    least = d.min(2, keepdims=True)
    near = d == least
    first, last = near.argmax(2), 7 - near[..., ::-1].argmax(2)
    code = np.where(first % 2 == 0, first, last)  # (of two neighbours one is even)
    code = code + 8 * np.signbit(v)
    return np.where(b == 255, 0, code).astype(np.uint8)


def pack(code):
    """Codes (..., C) to bytes (..., ceil(C / 2)), the first of a pair in the lower half."""
    if code.shape[-1] % 2:
        code = np.concatenate([code, np.zeros((*code.shape[:-1], 1), np.uint8)], -1)
    return code[..., 0::2] | code[..., 1::2] << 4


def quantize(v):
    s = scales(v)
    return pack(codes(v, s)), s


def values(packed, scale, cols):
    """What packed codes (..., bytes) stand for, (..., cols)."""
    code = np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], -1)[..., :cols]
    v = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
    s = np.repeat(scale, BLOCK, -1)[..., :cols].astype(float)
    with np.errstate(over="ignore"):
        return np.where(s == 255, np.nan, v * 2.0 ** (s - 127))


def silu(x):
    with np.errstate(over="ignore"):
        return x / (1 + np.exp(-x))


def layer(x, index, weight, w_in, w_out, first=0):
    """y = sum_k weight * W_out z, z = silu(gate) * up, over the held experts first, first + 1, ... And what errors are measured
    by: the same sum of sizes; the same of what a change of the gates' and ups' sums by their sums of sizes does to z
    (|d silu| <= 1.1); and the greatest gate."""
    T, C = x.shape
    F = w_out.shape[2]
    y, size, spread, greatest = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C)), 0.0
    for t in range(T):
        for k in range(index.shape[1]):
            e = index[t, k] - first
            if index[t, k] < 0 or not 0 <= e < w_in.shape[0]:
                continue
            h = w_in[e] @ x[t]
            mag = np.abs(w_in[e]) @ np.abs(x[t])
            g, u = h[:F], h[F:]
            z = silu(g) * u
            dz = 1.1 * mag[:F] * np.abs(u) + np.abs(silu(g)) * mag[F:]
            y[t] += weight[t, k] * (w_out[e] @ z)
            size[t] += abs(weight[t, k]) * (np.abs(w_out[e]) @ np.abs(z))
            spread[t] += abs(weight[t, k]) * (np.abs(w_out[e]) @ dz)
            greatest = max(greatest, np.abs(g).max(initial=0))
    return y, size, spread, greatest
