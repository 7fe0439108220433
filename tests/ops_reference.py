"""Plain 64-bit forms of the operators of include/gecc_ops.h, written from their definitions in numpy; shares no code with the
GPU path."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """Nearest bfloat16, ties to even, as float32 (finite values)."""
    u = np.asarray(x, np.float32).view(np.uint32)
    r = ((u >> 16) & 1) + 0x7fff
    out = ((u + r) & np.uint32(0xffff0000)).view(np.float32)
    return np.where(np.isfinite(x), out, np.asarray(x, np.float32))


def quantise(x):
    """x [rows, cols] -> codes [rows, cols] (sign << 3 | code), scale bytes [rows, blocks]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    p = np.zeros((rows, nb * 32))
    p[:, :cols] = x
    p = p.reshape(rows, nb, 32)
    bad = ~np.isfinite(p).all(axis=2)
    p = np.where(bad[:, :, None], 0.0, p)
    amax = np.abs(p).max(axis=2)
    e = np.where(amax > 0, np.frexp(amax)[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    v = np.ldexp(p, -e[:, :, None])
    d = np.abs(np.abs(v)[..., None] - GRID)                     # exact: few bits
    best = d.min(axis=3, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(axis=3), even.argmax(axis=3), near.argmax(axis=3))
    code = code | (np.signbit(p) << 3)
    return code.reshape(rows, -1)[:, :cols].astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales):
    rows, cols = codes.shape
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(s, 32, axis=1)[:, :cols]


def rounded(x):
    return values(*quantise(x))


def packed(codes, scales):
    """The two buffers of the library."""
    rows, cols = codes.shape
    P = -(-cols // 256) * 256
    c = np.zeros((rows, P), np.uint8)
    c[:, :cols] = codes
    data = c[:, 0::2] | (c[:, 1::2] << 4)
    units, r16 = -(-P // 512), -(-rows // 16)
    s = np.zeros((r16 * 16, units * 16), np.uint8)
    s[:rows, :scales.shape[1]] = scales
    out = np.zeros((r16, units, 16, 4, 4), np.uint8)
    for blk in range(16):
        out[:, :, :, blk % 4, blk // 4] = s.reshape(r16, 16, units, 16)[:, :, :, blk].transpose(0, 2, 1)
    return data, out


def orthogonalise(g, momentum, mu, nesterov, steps, coefficients, eps, scale):
    """(O, the momentum after), through the singular values: sigma -> a sigma + b sigma^3 + c sigma^5, `steps` times."""
    g = np.asarray(g, np.float64)
    m = None
    if momentum is not None:
        m = mu * np.asarray(momentum, np.float64) + g
        g = g + mu * m if nesterov else m
    x = g / (np.sqrt((g * g).sum()) + eps)
    u, s, vt = np.linalg.svd(x, full_matrices=False)
    a, b, c = coefficients
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return scale * (u * s) @ vt, m
