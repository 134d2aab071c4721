"""Float64 reference of the paged key/value cache and of attention over it (test infrastructure only; shares no code with the library).

  bf16            round to nearest even to bf16, as float64
  quantise        Appendix B's zero-point quantiser with 4 bits per row, range widened to hold 0, step rounded to bf16
  block_bytes, pack, unpack   one page's block for one head, as documented in include/conqur.h
  attend          softmax attention of query rows over the positions each one sees
"""
import numpy as np

NIBBLE_ELEMENT = [0, 2, 4, 6, 1, 3, 5, 7]


def bf16_bits(x):
    b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16)).astype(np.uint16)
    return np.where(np.isnan(np.asarray(x, dtype=np.float32)), np.uint16(0x7FC0), r)


def bits_value(b):
    return (np.asarray(b, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def bf16(x):
    return bits_value(bf16_bits(x))


def quantise(y, clip=1.0):
    """y (..., d) values of bf16.  Returns (codes, zero-point codes (..., 1), step (..., 1)); a row with a value not finite or of 2^127 or more has step NaN."""
    y = np.asarray(y, dtype=np.float64)
    c = float(np.float32(clip))
    odd = ~(np.abs(y) < 2.0 ** 127).all(axis=-1, keepdims=True)
    y = np.where(odd, 0.0, y)
    lo, hi = c * np.minimum(y.min(axis=-1, keepdims=True), 0.0), c * np.maximum(y.max(axis=-1, keepdims=True), 0.0)
    step = bf16((hi - lo) / 15.0)
    step = np.where(step < 2.0 ** -100, 0.0, step)
    by = np.where(step > 0, step, 1.0)
    zero = np.where(step > 0, np.clip(-np.rint(lo / by), 0, 15), 0.0)
    codes = np.where(step > 0, np.clip(np.rint(y / by) + zero, 0, 15), 0.0)
    return codes, zero, np.where(odd, np.nan, step)


def values(y, bits, clip=1.0):
    """What the cache holds of rows y."""
    if bits == 16:
        return np.asarray(y, dtype=np.float64)
    codes, zero, step = quantise(y, clip)
    return (codes - zero) * step


def block_bytes(page, d, bits):
    return page * (d + 8) if bits == 4 else 4 * page * d


def pack(k, v, page, bits, clip=1.0):
    """The bytes of one block from keys and values (page, d)."""
    d = k.shape[1]
    if bits == 16:
        out = []
        for y in (k, v):
            raw = bf16_bits(y)
            for plane in range(d // 64):
                rows = np.zeros((page, 64), np.uint16)
                for t in range(page):
                    for j in range(8):
                        rows[t, 8 * (j ^ (t & 7)):8 * (j ^ (t & 7)) + 8] = raw[t, 64 * plane + 8 * j:64 * plane + 8 * j + 8]
                out.append(rows.view(np.uint8).reshape(-1))
        return np.concatenate(out)
    codes, records = [], []
    for y in (k, v):
        c, z, s = quantise(y, clip)
        words = np.zeros((page, d // 8), np.uint32)
        for i, e in enumerate(NIBBLE_ELEMENT):
            words |= c[:, e::8].astype(np.uint32) << np.uint32(4 * i)
        codes.append(words.view(np.uint8).reshape(-1))
        records.append((bf16_bits(s[:, 0]).astype(np.uint32) | (z[:, 0].astype(np.uint32) << np.uint32(16))).view(np.uint8))
    return np.concatenate(codes + records)


def attend(q, k, v, seen, scale):
    """q (rows, d), k and v (positions, d), seen (rows, positions): (out, lse, sum of p |v|, largest sum of |q k| scale a row)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    out = np.zeros((q.shape[0], v.shape[1]))
    lse, mass, size = np.full(q.shape[0], -np.inf), np.zeros_like(out), np.zeros(q.shape[0])
    for i in range(q.shape[0]):
        at = np.flatnonzero(seen[i])
        if len(at) == 0:
            continue
        s = scale * (k[at] @ q[i])
        m = s.max()
        p = np.exp(s - m)
        total = p.sum()
        out[i], lse[i] = (p @ v[at]) / total, m + np.log(total)
        mass[i], size[i] = (p @ np.abs(v[at])) / total, abs(scale) * (np.abs(k[at]) @ np.abs(q[i])).max()
    return out, lse, mass, size
