"""Plain references of the 8-bit cache and of its pages, on the CPU: fixed sequences of fp32 operations where that is the
definition, whole numbers, or 64 bits, written apart from the kernels."""
import functools
import math

import numpy as np
import torch

F = np.float32


def sixteen(D):
    return 32 * D + 64


def key_at(D, t, c):
    """Where the code of channel c of token t's key lies in its sixteen."""
    chunk = c // 64
    if chunk < D // 64:
        return t // 4 * 4 * D + chunk * 256 + (c % 64 // 16 * 4 + t % 4) * 16 + c % 16
    return t // 4 * 4 * D + chunk * 256 + (c % 64 // 8 * 4 + t % 4) * 8 + c % 8


@functools.lru_cache(maxsize=None)
def key_order(D):
    return np.array([[key_at(D, t, c) for c in range(D)] for t in range(16)])


def empty(pages, H, page, D):
    return np.zeros((pages, H, page // 16, sixteen(D)), np.uint8)


def codes_of(block, D):
    """Bytes [..., 32 D + 64] -> codes of keys and values [..., 16, D] (whole numbers) and the two factors [..., 2]."""
    k = block[..., key_order(D)].astype(np.int32) - 128
    v = block[..., 16 * D:32 * D].reshape(*block.shape[:-1], D, 16).swapaxes(-1, -2).astype(np.int32) - 128
    return k, v, np.ascontiguousarray(block[..., 32 * D:32 * D + 8]).view(np.float32)


def put(block, D, k, v, q):
    """Its inverse."""
    block[..., key_order(D)] = (k + 128).astype(np.uint8)
    block[..., 16 * D:32 * D] = (v + 128).astype(np.uint8).swapaxes(-1, -2).reshape(*block.shape[:-1], -1)
    block[..., 32 * D:32 * D + 8] = np.ascontiguousarray(q, dtype=np.float32).view(np.uint8)


def finite_abs(x):
    return np.where(np.isfinite(x), np.abs(x), 0).astype(np.float32)


def quantize(r, q):
    with np.errstate(all="ignore"):
        z = np.clip(np.rint(r / (q if q > 0 else F(1))), -128, 127)
    return np.where(np.isnan(r), 0, z).astype(np.int32)


def write(cache, k, v, slots, page):
    """k, v: fp32 numpy [T, H, D]; into cache (uint8 numpy [pages, H, page / 16, 32 D + 64]), sixteen by sixteen."""
    pages, H, _, width = cache.shape
    D = (width - 64) // 32
    groups = {}
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            groups.setdefault(int(s) // 16, {})[int(s) % 16] = t
    for g, tokens in groups.items():
        places = sorted(tokens)
        rows = [tokens[i] for i in places]
        for h in range(H):
            block = cache[g * 16 // page, h, g * 16 % page // 16]
            zk, zv, q = codes_of(block, D)
            z, q = [zk, zv], q.copy()
            for i, x in enumerate((k, v)):
                r = x[rows, h]
                need = finite_abs(r).max() * (F(1) / F(127))
                if places[0] == 0:
                    z[i][:] = 0
                    q[i] = need
                elif need > q[i]:
                    new = max(need, F(1.25) * q[i])
                    z[i] = np.rint(z[i].astype(np.float32) * (q[i] / new)).astype(np.int32)
                    q[i] = new
                assert need.dtype == np.float32
                z[i][places] = quantize(r, q[i])
            put(block, D, z[0], z[1], q)


def read(cache, slots, page):
    """-> fp32 keys and values [T, H, D] (a code times its factor, one fp32 product)."""
    pages, H, _, width = cache.shape
    D = (width - 64) // 32
    out = np.zeros((2, len(slots), H, D), np.float32)
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            zk, zv, q = codes_of(cache[s // page, :, s % page // 16], D)
            out[0, t] = zk[:, s % 16].astype(np.float32) * q[:, :1]
            out[1, t] = zv[:, s % 16].astype(np.float32) * q[:, 1:]
    return out


def held(cache, table, b, length, page):
    """Keys and values of request b in 64 bits, [length, H, D]."""
    D = (cache.shape[3] - 64) // 32
    n = -(-length // 16)
    if n == 0:
        return np.zeros((2, 0, cache.shape[1], D))
    at = np.arange(n) * 16
    zk, zv, q = codes_of(cache[table[b, at // page], :, at % page // 16], D)             # [n, H, 16, D], [n, H, 2]
    kv = [(z * q[..., i, None, None].astype(np.float64)).transpose(0, 2, 1, 3).reshape(n * 16, -1, D)[:length]
          for i, z in enumerate((zk, zv))]
    return kv


def attend(q, keys, values, lengths, starts, scale, window=0, causal=True):
    """q: fp64 [T, heads * ratio, D]; keys, values: fp64 per request [length, heads, D].  -> out, and for every row and
    head the largest sum of |q k| scale and of |k| max|q| scale over seen keys."""
    out = np.zeros_like(q)
    noise = np.zeros(q.shape[:2] + (2,))
    for b, n_keys in enumerate(lengths):
        rows = slice(starts[b], starts[b + 1])
        n = starts[b + 1] - starts[b]
        behind = np.arange(n_keys)[None] - (np.arange(n) + n_keys - n)[:, None]              # of a key to a row's own
        seen = (behind <= 0) & (behind > -window if window else True) if causal else np.ones((n, n_keys), bool)
        for h in range(q.shape[1] if n and n_keys else 0):
            k, v = keys[b][:, h * keys[b].shape[1] // q.shape[1]], values[b][:, h * keys[b].shape[1] // q.shape[1]]
            s = np.where(seen, q[rows, h] @ k.T * scale, -np.inf)
            p = np.exp(s - np.where(seen.any(1), s.max(1), 0)[:, None])
            out[rows, h] = p @ v / np.maximum(p.sum(1), 1e-300)[:, None]
            noise[rows, h, 0] = np.where(seen, np.abs(q[rows, h]) @ np.abs(k).T, 0).max(1) * abs(scale)
            noise[rows, h, 1] = np.abs(q[rows, h]).max(1) * np.abs(k).sum(1).max() * abs(scale)
    return out, noise


def tolerance(out, noise, values, dtype):
    """How far the kernels may be off, element by element.  Keys are multiplied as codes, exactly; a query is scaled by a power
    of two and exact, unless it is 2^-14 of its row's largest or less: then it is off by 2^-25 of that.  Sums of the matrix
    instruction are of fp32 terms cut at the largest addend, in steps of 32 (2^-20 of the sum of magnitudes).  A score is
    off by d at most, which moves weights by a factor of exp(2 d).  A probability times its sixteen's factor is rounded once (2^-11),
    or off by 2^-25 / 2^3 of the largest such product where it is below binary16's normal numbers; a sum of n fp32 terms is off by
    n 2^-24 of it, the exponential by 2^-22, the output's own rounding by half a step of its type."""
    d = noise[..., 0] * 2.0 ** -20 + noise[..., 1] * 2.0 ** -25
    n = max([len(v) for v in values] or [0])
    top = max([np.abs(v).max() for v in values if v.size] or [0.0])
    rel = np.expm1(2 * d) + 2.0 ** -11 + n * (2.0 ** -27 + 2.0 ** -24) + 2.0 ** -21
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -11
    # (fp16 below 2^-14: steps of 2^-24)
    return top * rel[..., None] + np.abs(out) * half + (2.0 ** -25 if dtype is torch.float16 else 0.0)


def norm_bound(want, dtype):
    """What |off| over all outputs (a norm) is expected to stay below: a rounding to a type whose unit at 1 is u is off by u /
    sqrt(12) in the root mean square at most; the probabilities' (binary16) and the outputs' add up as squares.  fp16
    outputs that are subnormal are off by 2^-25."""
    half, own = 2.0 ** -10 / math.sqrt(12), (2.0 ** -7 if dtype is torch.bfloat16 else 2.0 ** -10) / math.sqrt(12)
    subnormal = 2.0 ** -25 * math.sqrt(want.size) if dtype is torch.float16 else 0.0
    return math.sqrt(half ** 2 + own ** 2) * np.linalg.norm(want) + subnormal


def pages_held(tokens, page, width):
    return -(-min(max(tokens, 0), width * page) // page)


def select(parents, lengths, table, page, n_pages):
    n, width = table.shape
    out = np.full((len(parents), width), -1, np.int32)
    lens, used, wants, seen = [], set(), [], set()
    for c, b in enumerate(parents):
        if not 0 <= b < n:
            lens.append(0)
            continue
        length = min(max(lengths[b], 0), width * page)
        held = pages_held(length, page, width)
        lens.append(length)
        out[c, :held] = table[b, :held]
        if b in seen:
            if length % page:
                wants.append(c)
        else:
            used.update(int(x) for x in table[b, :held] if 0 <= x < n_pages)
        seen.add(b)
    free = [x for x in range(n_pages) if x not in used]
    copies, refused, free = [], 0, free[::-1]
    for c in wants:
        if not free:
            refused += 1
            lens[c] = 0
            out[c] = -1
            continue
        last = lens[c] // page
        copies.append((int(out[c, last]), free.pop()))
        out[c, last] = copies[-1][1]
    counts, free = [len(free), len(copies), refused, n_pages - len(free)], free[::-1]
    return out, lens, free + [-1] * (n_pages - len(free)), copies + [(-1, -1)] * (len(parents) - len(copies)), counts


def compact(lengths, table, page, n_pages):
    n, width = table.shape
    held = [pages_held(t, page, width) for t in lengths]
    used = sorted({int(x) for b in range(n) for x in table[b, :held[b]] if 0 <= x < n_pages})
    k = len(used)
    goes, takes = [x for x in used if x >= k], sorted(set(range(k)) - set(used))
    to = dict(zip(goes, takes))
    out = np.full((n, width), -1, np.int32)
    for b in range(n):
        out[b, :held[b]] = [to.get(int(x), int(x)) for x in table[b, :held[b]]]
    moves = list(zip(goes, takes))
    return (out, list(range(k, n_pages)) + [-1] * k, moves + [(-1, -1)] * (n_pages // 2 - len(moves)),
            [n_pages - k, len(moves), 0, k])
