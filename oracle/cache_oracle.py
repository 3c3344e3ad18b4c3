"""fp64 statements of the operators that fill a cache and read the blocks of it that queries select: rotation by position, the 4-bit
and 8-bit formats, the bounds of a block's keys, scores and selection, attention over listed blocks.

Plain loops on numpy arrays of values; no code is shared with the GPU path.
"""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3_values():
    """The 256 values of e4m3: sign, four bits of exponent (bias 7), three of fraction; S.1111.111 is NaN, there are no infinities."""
    out = []
    for bits in range(256):
        e, f = bits >> 3 & 15, bits & 7
        x = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out.append((-1 if bits & 128 else 1) * (np.nan if e == 15 and f == 7 else x))
    return np.array(out)


def to_e4m3(x):
    """Bits of the nearest e4m3 value (halfway: the even fraction), beyond 448 of 448."""
    pos = e4m3_values()[:127]
    x = np.asarray(x, np.float64)
    a = np.abs(np.where(np.isnan(x), 0, x))
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    down = a - pos[lo] < pos[hi] - a
    tie = a - pos[lo] == pos[hi] - a
    bits = np.where(down | (tie & (lo % 2 == 0)), lo, hi)
    bits = np.where(a >= 448, 126, bits)
    return np.where(np.isnan(x), 127, bits | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def fp4_values(codes, scales):
    """codes[..., D/2] (two a byte, the low half first) and scales[..., D/16] (e4m3) -> values[..., D]."""
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    x = np.where(nibbles & 8, -1.0, 1.0) * E2M1[nibbles & 7]
    return x * np.repeat(e4m3_values()[scales], 16, axis=-1)


def to_fp4(x):
    """x[..., D] (fp32 values) -> codes and scales: scale = e4m3(max |x| / 6) of each 16, codes to nearest, halfway to even; the two
    quotients are fp32."""
    g = np.asarray(x, np.float32).reshape(*x.shape[:-1], -1, 16)
    scales = to_e4m3((np.abs(g).max(-1) / np.float32(6)).astype(np.float32))
    s = e4m3_values()[scales].astype(np.float32)[..., None]
    with np.errstate(all="ignore"):
        z = np.where(s == 0, np.float32(0), g / s).astype(np.float64)
    a = np.abs(z)[..., None]
    distance = np.abs(np.minimum(a, 6.0) - E2M1)
    best = distance.min(-1, keepdims=True)
    even = np.where(distance == best, np.arange(8) % 2, 9)     # of the nearest, the one with an even fraction
    code = np.argmin(even, -1).astype(np.uint8) | np.where(np.signbit(z), 8, 0).astype(np.uint8)
    code = code.reshape(*x.shape)
    return (code[..., ::2] | code[..., 1::2] << 4).astype(np.uint8), scales


def rotated(x, angles, cos_sin, interleaved):
    """x[..., t, D], the row of token t rotated by cos_sin[angles[t]] (cosines, then sines); fp64, then fp32."""
    x = x.astype(np.float64).copy()
    R = 0 if cos_sin is None else cos_sin.shape[1]
    for i in range(R // 2):
        a, z = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        c, s = cos_sin[angles, i].astype(np.float64), cos_sin[angles, R // 2 + i].astype(np.float64)
        x[..., a], x[..., z] = x[..., a] * c - x[..., z] * s, x[..., z] * c + x[..., a] * s
    return x.astype(np.float32)


def bounds(k, n, block):
    """k[T, D] of one head -> least, most [ceil(n / block), D]."""
    parts = [k[j: min(n, j + block)] for j in range(0, n, block)]
    return np.array([p.min(0) for p in parts]), np.array([p.max(0) for p in parts])


def scores(q, least, most):
    """q[group, D], bounds [m, D] -> [m]."""
    return np.maximum(q[:, None] * least, q[:, None] * most).sum((0, 2))


def attention(q, K, V, positions, scale):
    """q[group, D] over the rows `positions` (repeats count again) -> out, lse, sum of weight |v|, largest scale sum |q||k|."""
    K, V = K[positions].astype(np.float64), V[positions].astype(np.float64)
    if len(positions) == 0:
        return np.zeros(q.shape), np.full(q.shape[0], -np.inf), np.zeros(q.shape), 0.0
    s = scale * (q @ K.T)
    top = s.max(1, keepdims=True)
    p = np.exp(s - top)
    total = p.sum(1, keepdims=True)
    p /= total
    return p @ V, (top + np.log(total))[:, 0], p @ np.abs(V), float((scale * (np.abs(q) @ np.abs(K).T)).max())
