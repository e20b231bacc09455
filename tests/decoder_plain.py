"""Plain references of the operators on rows and on the 4-bit cache, on the CPU: the definitions in 64 bits (or, where
the result is a fixed sequence of fp32 operations, in exactly those), written apart from the kernels."""
import math

import numpy as np
import torch

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def finite_abs(x):
    return np.where(np.isfinite(x), np.abs(x), 0).astype(np.float32)


def quantize_rows(x):
    """x: torch [M, K] of any type -> (codes int8, factors fp32), fp32 step by step."""
    v = x.float().numpy()
    with np.errstate(all="ignore"):
        q = finite_abs(v).max(1) * (np.float32(1) / np.float32(127))
        q = np.where(q > 0, q, np.float32(1)).astype(np.float32)
        z = np.clip(np.rint(v / q[:, None]), -128, 127)
    return np.where(np.isnan(v), 0, z).astype(np.int8), q


def linear(z, q_x, z_w, q_w, bias, dtype):
    """The exact sum, then the stated fp32 operations, rounded to dtype."""
    acc = (torch.from_numpy(z).double() @ torch.from_numpy(z_w).double().t()).numpy()      # (exact: below 2^53)
    y = acc.astype(np.float32) * (q_x[:, None] * q_w[None, :])
    if bias is not None:
        y = y + bias
    assert y.dtype == np.float32
    return torch.from_numpy(y).to(dtype)


def page_tables(lengths, added, page, free, table, n_slots):
    """One request after the other."""
    table = table.copy()
    starts, grown, slots, positions = [0], [], [-1] * n_slots, [-1] * n_slots
    upto = taken = refused = 0
    for b, (n, a) in enumerate(zip(lengths, added)):
        n, a = max(n, 0), max(a, 0)
        first, end = starts[-1], starts[-1] + a
        starts.append(end)
        have, total = -(-n // page), -(-(n + a) // page)
        fits = total <= table.shape[1] and end <= n_slots
        if fits:
            upto += total - have
            fits = total == have or upto <= len(free)
        if not fits:
            refused += 1
            grown.append(n)
            continue
        for i in range(have, total):
            table[b, i] = free[upto - total + i]
        taken += total - have
        grown.append(n + a)
        for i in range(a):
            slots[first + i] = int(table[b, (n + i) // page]) * page + (n + i) % page
            positions[first + i] = n + i
    return table, slots, positions, starts, grown, [taken, starts[-1], refused]


def kv4_codes(x):
    """x: fp32 numpy [..., D] -> (codes -8 .. 7 [..., D], factors binary16 [..., D / 32])."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    with np.errstate(all="ignore"):
        q = np.minimum(finite_abs(g).max(-1) * (np.float32(1) / np.float32(7)), np.float32(8188)).astype(np.float16)
        q = np.where(q == 0, np.float16(1), q)
        z = np.clip(np.rint(g / q.astype(np.float32)[..., None]), -8, 7)
    return np.where(np.isnan(g), 0, z).astype(np.int8).reshape(x.shape), q


def kv4_write(cache, k, v, slots, page):
    """Byte by byte into cache (uint8 numpy [pages, heads, page / 16, 18 D]), by the layout."""
    pages, H, _, width = cache.shape
    D = width // 18
    G = D // 32
    zk, qk = kv4_codes(k)
    zv, qv = kv4_codes(v)
    for t, slot in enumerate(slots):
        if not 0 <= slot < pages * page:
            continue
        for h in range(H):
            b = cache[slot // page, h, slot % page // 16]
            at = int(slot % 16)
            place = (at & ~3) + [0, 2, 1, 3][at & 3]
            for g in range(G):
                for j in range(4):
                    for i in range(0, 8, 2):
                        c = 32 * g + 8 * j + i
                        b[at * 16 * G + j * 4 * G + 4 * g + i // 2] = zk[t, h, c] + 8 | zk[t, h, c + 1] + 8 << 4
                for r in range(16):
                    c = 32 * g + r
                    b[256 * G + (g * 16 + r) * 16 + at] = zv[t, h, c] + 8 | zv[t, h, c + 16] + 8 << 4
                b[512 * G + 2 * (at * G + g):][:2] = np.frombuffer(qk[t, h, g].tobytes(), np.uint8)
                b[544 * G + 2 * (g * 16 + place):][:2] = np.frombuffer(qv[t, h, g].tobytes(), np.uint8)


def kv4_values(x):
    """What the cache holds for fp32 values x [..., D], in fp64 (a code times its factor)."""
    z, q = kv4_codes(x)
    return z.astype(np.float64) * np.repeat(q.astype(np.float64), 32, -1)


def attend(q, keys, values, lengths, starts, scale, window):
    """q: fp64 [T, heads * ratio, D]; keys, values: fp64 per request [length, heads, D].  -> (out, the largest
    sum of |q k| scale over seen keys)"""
    out = np.zeros_like(q)
    most = 0.0
    for b, n_keys in enumerate(lengths):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            pos = n_keys - n + i
            lo = max(0, pos - window + 1) if window else 0
            if pos < lo or pos < 0:
                continue
            ratio = q.shape[1] // keys[b].shape[1]
            for h in range(q.shape[1]):
                row, k = q[starts[b] + i, h], keys[b][lo:pos + 1, h // ratio]
                s = k @ row * scale
                most = max(most, float((np.abs(k) @ np.abs(row)).max() * scale))
                p = np.exp(s - s.max())
                out[starts[b] + i, h] = (p / p.sum()) @ values[b][lo:pos + 1, h // ratio]
    return out, most


def attend_tolerance(out, values, most, dtype):
    """How far the kernel may be off, element by element.  Its products are of binary16 numbers: a key or a value is a
    code times its factor rounded once (2^-11 of it at most), a query is scaled by a power of two and exact in fp16 and
    bf16 alike unless it is 2^-14 of its row's largest (then off by 2^-25 of that).  (For bf16 outputs of many rows the queries have the scale in
    them and are rounded too: nothing is added for that, since it and the keys' rounding are the worst case of 2^-11 in
    each of D products, all of one sign.)  A score is then off by at most
    d = 2^-11 sum |q k| scale (and fp32 noise, 2^-20 of the same), which moves weights by a factor of exp(2 d) at most; a
    probability is rounded once more (2^-11) while the sum of them is not, and a probability below 2^-14 of the
    largest is off by 2^-25.  The output is rounded once."""
    d = most * (2.0 ** -11 + 2.0 ** -20)
    n = max(len(v) for v in values)
    top = max([np.abs(v).max() for v in values if v.size] or [0.0])
    rel = math.expm1(2 * d) + 2.0 ** -11 + 2.0 ** -11 + n * 2.0 ** -25
    return top * rel + np.abs(out) * (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -11) + 1e-7 * top


def attend_rows(q, keys, values, lengths, starts, scale, window=0):
    """As ``attend``, a head of a request at a time: for many rows."""
    out = np.zeros_like(q)
    for b, n_keys in enumerate(lengths):
        rows = slice(starts[b], starts[b + 1])
        n = starts[b + 1] - starts[b]
        ratio = q.shape[1] // keys[b].shape[1]
        behind = np.arange(n_keys)[None] - (np.arange(n) + n_keys - n)[:, None]              # of a key to a row's own
        seen = (behind <= 0) & (behind > -window if window else True)
        for h in range(q.shape[1] if n and n_keys else 0):
            s = np.where(seen, q[rows, h] @ keys[b][:, h // ratio].T * scale, -np.inf)
            p = np.exp(s - np.where(seen.any(1), s.max(1), 0)[:, None])
            out[rows, h] = p @ values[b][:, h // ratio] / np.maximum(p.sum(1), 1e-300)[:, None]
    return out


def attend_norm(want, dtype, wide, spread):
    """What |off| over all outputs (a norm) is expected to stay below.  A rounding to a type whose unit at 1 is u is off by
    at most u / sqrt(12) of a value in the root mean square (by as little as half of that where the value is just below a
    power of two), and roundings of different numbers are independent: their squares add up.
      tiles of 16 columns    a probability times its token's factor is rounded to binary16, the output to its type
      tiles of 128 columns   a value (code times factor) and a probability to binary16, the output to its type
        bf16                 ... and a key and a query, channel by channel: a score is then off by that of what scores
                             spread by, and a probability by as much of itself
    Outputs in fp16 are off by 2^-25 where they are subnormal."""
    half, own = 2.0 ** -10 / math.sqrt(12), (2.0 ** -7 if dtype is torch.bfloat16 else 2.0 ** -10) / math.sqrt(12)
    squares = own ** 2 + half ** 2 * (2 if wide else 1)
    if wide and dtype is torch.bfloat16:
        squares += 2 * (spread * half) ** 2
    subnormal = 2.0 ** -25 * math.sqrt(want.size) if dtype is torch.float16 else 0.0
    return math.sqrt(squares) * np.linalg.norm(want) + subnormal
