"""64-bit forms of the 4-bit cache of keys and values and of few rows times 4-bit weights (numpy, CPU): written from the
definitions in include/svg.h, sharing nothing with the library."""
import math

import numpy as np

from . import block_oracle as B


def record_bytes(D, page_size):
    return page_size * (D + D // 16)


def parts(D, page_size):
    """Where the parts of a record begin, and the bytes of a token in each: keys, values, keys' scales, values' scales."""
    starts = np.cumsum([0, page_size * (D // 2), page_size * (D // 2), page_size * (D // 32)])
    return list(zip(starts.tolist(), (D // 2, D // 2, D // 32, D // 32)))


def write(data, k, v, slots, page_size):
    """data uint8 [pages, H, record]; k, v [rows, H, D] in 64 bits; slots outside of the pool are skipped."""
    pages, H, _ = data.shape
    rows, _, D = k.shape
    for (start, size), (scale_start, scale_size), x in zip(parts(D, page_size)[:2], parts(D, page_size)[2:], (k, v)):
        codes, scales = B.mx_quantise(x.reshape(rows * H, D))
        packed = (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8).reshape(rows, H, D // 2)
        scales = scales.reshape(rows, H, D // 32)
        for m, slot in enumerate(slots):
            page, place = divmod(int(slot), page_size)
            if 0 <= slot and page < pages:
                data[page, :, start + place * size:start + (place + 1) * size] = packed[m]
                data[page, :, scale_start + place * scale_size:scale_start + (place + 1) * scale_size] = scales[m]


def read(data, slots, D, page_size):
    """(k, v) [rows, H, D] in 64 bits; NaN where the slot is outside of the pool."""
    pages, H, _ = data.shape
    out = []
    for (start, size), (scale_start, scale_size) in zip(parts(D, page_size)[:2], parts(D, page_size)[2:]):
        x = np.full((len(slots), H, D), np.nan)
        for m, slot in enumerate(slots):
            page, place = divmod(int(slot), page_size)
            if 0 <= slot and page < pages:
                packed = data[page, :, start + place * size:start + (place + 1) * size]
                codes = np.stack([packed & 15, packed >> 4], -1).reshape(H, D)
                x[m] = B.mx_values(codes, data[page, :, scale_start + place * scale_size:scale_start + (place + 1) * scale_size])
        out.append(x)
    return out


def seen(n, q_n, i, block, causal, window, sink):
    """Which of n tokens query i of q_n sees, by the definition, one comparison after the other."""
    p = n - q_n + i
    own = math.floor(p / block)
    j = np.arange(n)
    at = j // block
    yes = np.ones(n, dtype=bool)
    if causal:
        yes &= at <= own
    if window >= 0:
        yes &= (at >= own - window) | (j < sink)
    return yes


def attention(q, k, v, exists, scale, block=1, causal=False, window=-1, sink=0, q_n=None):
    """q [Hq, N, D], k and v [n, H, D] in 64 bits -> (o, lse, size, slack): size = the weighted mean of |v|, the magnitude that o is added
    up from, slack = the largest sum of |q k| times the scale, the magnitude that a score is added up from."""
    Hq, N, D = q.shape
    n, H, _ = k.shape
    q_n = N if q_n is None else q_n
    o, size = np.zeros((Hq, q_n, D)), np.zeros((Hq, q_n, D))
    lse, slack = np.full((Hq, q_n), -np.inf), np.zeros((Hq, q_n))
    for i in range(q_n):
        yes = np.nonzero(seen(n, q_n, i, block, causal, window, sink) & exists)[0]
        if not len(yes):
            continue
        for h in range(Hq):
            kk, vv = k[yes, h // (Hq // H)], v[yes, h // (Hq // H)]
            s = kk @ q[h, i] * scale
            top = s.max()
            e = np.exp(s - top)
            total = e.sum()
            lse[h, i] = top + np.log(total)
            o[h, i] = e @ vv / total
            size[h, i] = e @ np.abs(vv) / total
            slack[h, i] = (np.abs(kk) @ np.abs(q[h, i])).max() * scale
    return o, lse, size, slack


OK, FULL, LENGTHS, PAGES = 0, 1, 2, 3


def resize(table, lengths, wanted, free, count, page_size, tokens, with_slots=True):
    """(table, free, new_lengths, new_count, slots, status): lists walked one page after the other.  Entries outside of the pool are pages that
    are not there: nothing to give back, and never granted."""
    Bn, max_pages = table.shape
    most, pages = max_pages * page_size, len(free)
    none = np.full((Bn, tokens), -1, dtype=np.int64)
    refused = lambda why: (table.copy(), free.copy(), lengths.copy(), count, none, why)  # noqa: E731
    if any(not 0 <= a <= most or not 0 <= b <= most or (with_slots and b - a > tokens) for a, b in zip(lengths, wanted)):
        return refused(LENGTHS)
    if not 0 <= count <= pages:
        return refused(LENGTHS)
    held, need = -(-lengths // page_size), -(-wanted // page_size)
    back = [int(table[b, j]) for b in range(Bn) for j in range(need[b], held[b]) if 0 <= table[b, j] < pages]
    if count + len(back) > pages:
        return refused(LENGTHS)
    stack = [int(x) for x in free[:count]] + back
    new_free, new_table = free.copy(), table.copy()
    new_free[:len(stack)] = stack
    for b in range(Bn):
        for j in range(held[b], need[b]):
            if not stack:
                return refused(FULL)
            new_table[b, j] = stack.pop()
    if any(not 0 <= new_table[b, j] < pages for b in range(Bn) for j in range(held[b], need[b])):
        return refused(PAGES)
    slots = none
    for b in range(Bn):
        for i in range(min(tokens, max(0, wanted[b] - lengths[b]))):
            page, place = new_table[b, (lengths[b] + i) // page_size], (lengths[b] + i) % page_size
            slots[b, i] = page * page_size + place if 0 <= page < pages else -1
    return new_table, new_free, wanted.copy(), len(stack), slots, OK
