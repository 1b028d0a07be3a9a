"""Plain CPU oracle of rotary positions, of a cache in microscaled 4-bit elements and of the attention over it: the definitions in 64 bits over numpy arrays.
Shares no code with the library."""
import math

import numpy as np

from oracle import mx_oracle as mx


def rotate(x, positions, frequencies, rotary, pairs, transposed=False, factor=1.0):
    """x (T, H, D), positions (T), frequencies (rotary / 2) -> the result and what its errors scale with: the sums of |a c| + |b s|."""
    x = np.asarray(x, np.float64)
    y, size = x.copy(), np.zeros_like(x)
    for t in range(x.shape[0]):
        for i in range(rotary // 2):
            angle = float(int(positions[t])) * float(frequencies[i])   # at most 53 bits for what the tests take: exact
            c, s = factor * math.cos(angle), factor * math.sin(angle) * (-1 if transposed else 1)
            p, q = (i, i + rotary // 2) if pairs == "half" else (2 * i, 2 * i + 1)
            a, b = x[t, :, p], x[t, :, q]
            y[t, :, p], y[t, :, q] = a * c - b * s, b * c + a * s
            size[t, :, p], size[t, :, q] = abs(a * c) + abs(b * s), abs(b * c) + abs(a * s)
    return y, size


def read_slots(codes, codes_text, scales, scales_text, slots):
    """Values (len(slots), H, P) in 64 bits of the slots named."""
    q, s = mx.mode_offsets(codes_text), mx.mode_offsets(scales_text)
    off = q[0][slots][:, None, None] + q[1][None, :, None] + q[2][None, None, :]
    nibble = (codes[off // 2] >> (4 * (off % 2)).astype(np.uint8)) & 15
    byte = scales[s[0][slots][:, None, None] + s[1][None, :, None] + s[2][None, None, :]].astype(np.int64)
    scale = np.where(byte == 255, np.nan, np.ldexp(1.0, byte - 127))
    return mx.LEVELS[nibble] * np.repeat(scale, 32, axis=2)


def write_slots(codes, codes_text, scales, scales_text, slots, x, rule):
    """Quantises rows x (T, H, D) into the slots (those below 0 or beyond the last are left out); codes and scales are changed in place."""
    q, s = mx.mode_offsets(codes_text), mx.mode_offsets(scales_text)
    padded = len(q[2])
    for t, slot in enumerate(slots):
        if not 0 <= slot < len(q[0]):
            continue
        code, byte = mx.quantize(np.asarray(x[t], np.float64), padded, rule)
        for h in range(x.shape[1]):
            off = q[0][slot] + q[1][h] + q[2]
            for parity in (0, 1):
                at = off % 2 == parity
                where = off[at] // 2
                codes[where] = (codes[where] & (0xF0 if parity == 0 else 0x0F)) | (code[h][at].astype(np.uint8) << (4 * parity))
            scales[s[0][slot] + s[1][h] + s[2]] = byte[h]


def sequences(T, n_sequences, lengths, starts, page, pages_each, max_queries):
    """(first row of q, queries, position of the first query, length) of each, cut to what fits."""
    out = []
    for b in range(n_sequences):
        begin, end = (starts[b], starts[b + 1]) if starts is not None else (b * (T // n_sequences), (b + 1) * (T // n_sequences))
        begin = min(max(int(begin), 0), T)
        end = min(max(int(end), begin), T)
        length = min(max(int(lengths[b]), 0), page * pages_each)
        out.append((begin, min(end - begin, max_queries), length - (end - begin), length))
    return out


def attention(q, pool_k, pool_v, group, n_sequences, page, pages_each, max_queries, lengths, starts, pages, scale, causal, window, o, lse):
    """q (T, Hq, D); pool_k, pool_v: slots -> (len, Hkv, D) values.  Fills o (T, Hq, D) and lse (T, Hq) in place where there are queries, and returns (mass, spread):
    per element of o the weighted mean of |v|, and per row the largest |scale q k| sum and the smallest and number of what an error bound needs."""
    T, heads, D = q.shape
    mass, score_size, count = np.zeros(o.shape), np.zeros(lse.shape), np.zeros(lse.shape)
    loose = np.zeros(o.shape)
    for b, (first, n, position, length) in enumerate(sequences(T, n_sequences, lengths, starts, page, pages_each, max_queries)):
        j = np.arange(length)
        ids = np.asarray(pages[b])[j // page] if pages is not None else b * pages_each + j // page
        there = (ids >= 0) & (ids < pool_k.slots // page)
        slots = np.where(there, ids, 0) * page + j % page
        k, v = pool_k(slots), pool_v(slots)
        for i in range(n):
            seen = there & (j <= position + i if causal else j >= 0)
            if window:
                seen &= j > position + i - window
            for h in range(heads):
                ks, vs = k[seen, h // group], v[seen, h // group]
                row = first + i
                if not seen.any():
                    o[row, h], lse[row, h] = 0.0, -np.inf
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (ks @ q[row, h])
                    top = np.max(s) if not np.isnan(s).any() else np.nan
                    p = np.exp(s - top)
                    total = p.sum()
                    # (0 times an infinity is NaN, as it is for the matrix product)
                    o[row, h] = (p[:, None] * vs).sum(0) / total
                    lse[row, h] = top + np.log(total)
                    mass[row, h] = (p[:, None] * np.abs(vs)).sum(0) / total
                    loose[row, h] = np.abs(vs).sum(0) / total
                    score_size[row, h] = (abs(scale) * (np.abs(ks) @ np.abs(q[row, h]))).max()
                    count[row, h] = len(s)
    return mass, loose, score_size, count


class Pool:
    """One tensor of a cache: slots -> values of the first D elements."""

    def __init__(self, codes, codes_text, scales, scales_text, D):
        self.args, self.D = (codes, codes_text, scales, scales_text), D
        self.slots = len(mx.mode_offsets(codes_text)[0])

    def __call__(self, slots):
        return read_slots(*self.args, slots)[:, :, :self.D]
