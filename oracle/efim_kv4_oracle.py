"""CPU oracle of a step over a 4-bit KV cache: blocks of 4-bit floats, attention over them, block tables and slot maps, adjusted logits.

TEST INFRASTRUCTURE ONLY; shares no code with the library.  Everything in float64 (or whole numbers), as the definitions read.

Readings (the paper leaves model and cache as they are): a block is sixteen neighbouring dims of one token's head with a scale of
its own; e2m1 and e4m3 are the 4- and 8-bit floats whose values the tables below spell out; roundings are to nearest, ties to the even
code.  Penalties come in the order repetition, frequency, presence, bias, mask.
"""
import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])   # the last is NaN


def nearest(x, values):
    """Indexes of the nearest of some ascending values to x >= 0, of two alike the even one; the last for what is beyond it."""
    hi = np.clip(np.searchsorted(values, x), 1, len(values) - 1)
    down, up = x - values[hi - 1], values[hi] - x
    return np.where((down < up) | ((down == up) & (hi % 2 == 1)), hi - 1, hi)


def key(x, table, interleaved=False, weight=None, eps=0.0):
    """Heads x [..., D], normalised where there are weights and rotated by table rows [..., D] (cos, then sin; None: not), rounded to fp32, and that to bf16.
    -> numbers of 8 bits, as float64"""
    x, half = np.asarray(x, np.float64), x.shape[-1] // 2
    with np.errstate(all="ignore"):
        if weight is not None:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
        if table is not None:
            cos, sin = np.float64(table[..., :half]), np.float64(table[..., half:])
            a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
            x = np.stack([a * cos - b * sin, b * cos + a * sin], -1 if interleaved else -2).reshape(x.shape)
        bits = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    bits = np.where(np.isnan(x), 0x7fc00000, bits + 0x7fff + (bits >> 16 & 1) & 0xffff0000)
    return bits.astype(np.uint32).view(np.float32).astype(np.float64)


def quantize(x, g):
    """x: float64 [..., D], numbers with few bits (bf16).  -> codes uint8 [..., D / 2], scales uint8 [..., D / 16]."""
    x = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 16)
    with np.errstate(all="ignore"):
        y = x / g
        top = np.abs(y).max(-1)
        bad = np.isnan(top)
        # 6 s against the largest value: no quotient is rounded
        scale = np.maximum(nearest(np.where(bad, 0, np.minimum(top, 1e300)), 6 * E4M3), 1)
        code = nearest(np.minimum(np.abs(y), 1e300) / E4M3[scale][..., None], E2M1)     # (a quotient that is a border is exact)
    code = np.where(np.isnan(y), 7, code + np.where(np.signbit(y), 8, 0))
    code = code.reshape(*code.shape[:-2], -1)
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8), np.where(bad, 127, scale).astype(np.uint8)


def held(codes, scales, g):
    """Values that codes and scales stand for."""
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*scales.shape, 16).astype(np.int64)
    s = np.append(E4M3, np.nan)[scales & 127] * np.where(scales >= 128, -1, 1)
    return (np.where(code >= 8, -1, 1) * E2M1[code & 7] * s[..., None] * g).reshape(*codes.shape[:-1], -1)


def attend(q, k, v, limits, scale):
    """One kv head: q [rows, D], k and v [keys, D], row r sees keys below limits[r].  -> out, lse, the weighted mean of |v| and, per row,
    the largest sum of |q||k| over a key it sees (what the error bounds need).  Rows without keys: 0, -inf."""
    rows, d = q.shape
    out, size, lse, reach = np.zeros((rows, d)), np.zeros((rows, d)), np.full(rows, -np.inf), np.zeros(rows)
    for r in range(rows):
        n = min(max(int(limits[r]), 0), len(k))
        if n == 0:
            continue
        with np.errstate(all="ignore"):
            s = k[:n] @ q[r] * scale
            top = s.max()
            w = np.exp(s - top)
            out[r], size[r] = w @ v[:n] / w.sum(), w @ np.abs(v[:n]) / w.sum()
            lse[r] = top + np.log(w.sum())
            reach[r] = (np.abs(k[:n]) @ np.abs(q[r])).max() * scale
    return out, lse, size, reach


def step_tables(cached, new, table, free, room, page=16):
    """Lists of ints; table: list of lists; free: list, its last entry is taken first.  Sequences one after the other, places upwards.
    -> indptr, table, free, positions, slots, sequences (of `room` rows), whether pages ran out"""
    table, free, ran_out = [list(row) for row in table], list(free), False
    indptr, positions, slots, sequences = [0], [], [], []
    for s, (c, n) in enumerate(zip(cached, new)):
        for i in range(-(-c // page), -(-(c + n) // page)):
            if i < len(table[s]) and table[s][i] < 0:
                if free:
                    table[s][i] = free.pop()
                else:
                    ran_out = True
        for p in range(c, c + n):
            held_by = table[s][p // page] if p // page < len(table[s]) else -1
            positions.append(p)
            sequences.append(s)
            slots.append(held_by * page + p % page if held_by >= 0 else -1)
        indptr.append(indptr[-1] + n)
    pad = [-1] * max(0, room - len(positions))
    return indptr, table, free, (positions + pad)[:room], (slots + pad)[:room], (sequences + pad)[:room], ran_out


def adjust(x, prompt, output, repetition, frequency, presence, bias, allowed):
    """One row.  x: float64 [vocab]; prompt, output: token ids; bias: pairs (token, value), the last of a token counts; allowed: bool
    [vocab] or None.  -> the adjusted row and, per place, the sum of its terms' magnitudes"""
    x = np.array(x, np.float64)
    count = np.bincount(np.asarray(output, np.int64), minlength=len(x)).astype(np.float64)
    seen = count + np.bincount(np.asarray(prompt, np.int64), minlength=len(x)) > 0
    with np.errstate(all="ignore"):
        x = np.where(seen, np.where(x > 0, x / repetition, x * repetition), x)
        size = np.abs(x) + np.abs(frequency * count) + np.abs(presence * (count > 0))
        x = x - frequency * count - presence * (count > 0)
        for token, b in dict(bias).items():
            x[token] += b
            size[token] += abs(b)
    if allowed is not None:
        x[~allowed] = -np.inf
    return x, size
