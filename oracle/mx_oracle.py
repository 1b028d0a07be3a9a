"""Plain CPU oracle of microscaled 4-bit tensors: the definitions in 64 bits over numpy arrays, element by element in memory.
Shares no code with the library.  A matrix under a layout is read and written through the offsets of its rows and columns."""
import ast

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def _leaves(shape, stride):
    if isinstance(shape, tuple):
        return [leaf for s, d in zip(shape, stride) for leaf in _leaves(s, d)]
    return [(shape, stride)]


def mode_offsets(text):
    """Offsets of every coordinate of each top-level mode of "(..):(..)": L(r, k, ..) is the sum of one of each."""
    shape, stride = (ast.literal_eval(part) for part in text.split(":"))
    out = []
    for s, d in zip(shape, stride):
        off = np.zeros(1, np.int64)
        for extent, step in _leaves(s, d):   # leftmost leaf fastest
            off = (off[None, :] + np.arange(extent, dtype=np.int64)[:, None] * step).reshape(-1) if len(off) == 1 else \
                (np.arange(extent, dtype=np.int64)[:, None] * step + off[None, :]).reshape(-1)
        out.append(off)
    return out


def offsets(text):
    """Offsets of a layout of rank 2 (rows, columns) or 3 (rows, columns, batch)."""
    modes = mode_offsets(text)
    off = modes[0][:, None] + modes[1][None, :]
    return off if len(modes) == 2 else off[:, :, None] + modes[2][None, None, :]


def scale_bytes(largest, rule):
    """Block maxima (64 bits) -> scale bytes, from the definition: the exponent is searched, not computed from bits."""
    byte = np.zeros(largest.shape, np.int64)
    finite = np.isfinite(largest)
    for s in range(0, 255):
        p = np.ldexp(1.0, s - 127)
        if rule == "floor":   # the largest scale 2^e with 4 * 2^e <= a
            byte[finite & (4 * p <= largest)] = s
        else:                 # the smallest with a <= 6 * 2^e
            byte[finite & (largest > 6 * p)] = s + 1
    byte[~finite] = 255
    return byte


def nearest_codes(y):
    """|values| over their scale (64 bits) -> codes 0 .. 7: the nearest level, ties to the even code, 6 beyond the last."""
    distance = np.abs(np.minimum(y, 6.0)[..., None] - LEVELS[:8])
    best = distance.min(-1, keepdims=True)
    tied = distance == best
    even = tied & (np.arange(8) % 2 == 0)
    return np.where(even.any(-1), even.argmax(-1), tied.argmax(-1))


def quantize(x, padded, rule):
    """(R, K) values in 64 bits -> codes (R, padded) 0 .. 15, scale bytes (R, padded / 32)."""
    rows, k = x.shape
    v = np.zeros((rows, padded))
    v[:, :k] = x
    v = v.reshape(rows, padded // 32, 32)
    largest = np.abs(v).max(-1)
    largest[np.isnan(v).any(-1)] = np.nan
    byte = scale_bytes(largest, rule)
    bad = (byte == 255)[..., None]
    with np.errstate(invalid="ignore", over="ignore"):
        code = nearest_codes(np.where(bad, 0.0, np.abs(v) / np.ldexp(1.0, byte - 127)[..., None])) + 8 * np.signbit(v)
    return np.where(bad, 0, code).reshape(rows, padded), byte


def dequantize(codes, scale_byte):
    """codes (R, P), scale bytes (R, P / 32) -> values (R, P) in 64 bits."""
    scale = np.where(scale_byte == 255, np.nan, np.ldexp(1.0, scale_byte.astype(np.int64) - 127))
    return LEVELS[codes] * np.repeat(scale, 32, axis=1)


def put_codes(buf, text, codes):
    """Writes codes into the packed bytes of `buf` under a layout counted in 4-bit elements; other nibbles stay."""
    off = offsets(text)
    for parity in (0, 1):
        at = off % 2 == parity
        byte = off[at] // 2
        keep = buf[byte] & (0xF0 if parity == 0 else 0x0F)
        buf[byte] = keep | (codes[at].astype(np.uint8) << (4 * parity))


def get_codes(buf, text):
    off = offsets(text)
    return (buf[off // 2] >> (4 * (off % 2)).astype(np.uint8)) & 15
