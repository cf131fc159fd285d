"""Plain forms of the calls around the 8-bit cache, for the tests: one request, one block, one query at a time in numpy;
values in 64 bits, roundings of the definition in fp32."""
from __future__ import annotations

import numpy as np

F = np.float32


def places():
    """slot of place (half, i) of a tile's V rows"""
    return [[4 * h + i % 4 + 8 * (i // 4 % 2) + 16 * (i // 8) for i in range(16)] for h in range(2)]


class Cache:
    """The bytes of a cache as codes [n_blocks, S, H, d] of K and V and scales [n_blocks, H, 2], and back."""

    def __init__(self, data, n_blocks, S, H, d):
        e = -(-d // 16) * 16
        n = n_blocks * H * S * 2 * e
        assert data.dtype == np.uint8 and data.size == n + n_blocks * H * 8
        tiles = data[:n].reshape(n_blocks, H, S // 32, 64 * e)
        self.codes = [np.zeros((n_blocks, S, H, d), np.int64) for _ in range(2)]
        where = places()
        for t in range(S // 32):
            k = tiles[:, :, t, :32 * e].reshape(n_blocks, H, e // 16, 32, 16)
            v = tiles[:, :, t, 32 * e:].reshape(n_blocks, H, e, 2, 16)
            for x in range(d):
                self.codes[0][:, t * 32:t * 32 + 32, :, x] = np.moveaxis(k[:, :, x // 16, :, x % 16], 1, 2).astype(int) - 128
            for h in range(2):
                for i in range(16):
                    self.codes[1][:, t * 32 + where[h][i]] = v[:, :, :d, h, i].astype(int) - 128
        self.padding = [tiles[..., :32 * e].reshape(n_blocks, H, S // 32, e // 16, 32, 16)[:, :, :, -1, :, d - e + 16:],
                        tiles[..., 32 * e:].reshape(n_blocks, H, S // 32, e, 32)[:, :, :, d:]]
        self.scales = data[n:].view(F).reshape(n_blocks, H, 2).copy()
        self.S = S

    def values(self, which, block, slot):
        """fp32 [H, d] of one row, as it is defined: code * scale rounded once"""
        return self.codes[which][block, slot].astype(F) * self.scales[block, :, which][:, None]

    def exact(self, which, table, b, n):
        """[n, H, d] in 64 bits"""
        rows = [(table[b, r // self.S], r % self.S) for r in range(n)]
        return np.stack([self.codes[which][i, s] * self.scales[i, :, which].astype(np.float64)[:, None] for i, s in rows])


def plan(lengths, new, table, free, n_free, S, rows):
    """-> table, lengths, n_free, offsets, runs, counts"""
    B, W = table.shape
    table, out, left = table.copy(), list(lengths), max(0, min(int(n_free), len(free)))
    offsets, runs, asked, taken, refused = [0], [], 0, 0, 0
    for b in range(B):
        old, add = int(lengths[b]), int(new[b])
        offsets.append(offsets[-1] + max(add, 0))
        ok = old >= 0 and add >= 0 and old + add <= W * S and offsets[-1] <= rows
        need = (-(-(old + add) // S) - -(-old // S)) if ok else 0
        asked += need
        if not ok or (add and asked > left):
            refused += 1
            continue
        for c in range(-(-old // S), -(-old // S) + need):
            table[b, c] = free[left - 1 - taken]
            taken += 1
        out[b] = old + add
        at = old
        while at < old + add:
            end = min(old + add, at // S * S + S)
            runs.append((table[b, at // S], offsets[b] + at - old, at % S, end - at))
            at = end
    return table, out, left - taken, offsets, runs, [len(runs), taken, refused, offsets[-1]]


def release(done, lengths, table, free, n_free, S):
    """-> free list (its first entries), lengths"""
    free, W = list(free[:n_free]), table.shape[1]
    for b in range(len(lengths)):
        if done[b]:
            free += [int(x) for x in table[b, :min(W, -(-max(int(lengths[b]), 0) // S))]]
    return free, [0 if d else int(n) for d, n in zip(done, lengths)]


def quantize(x, old):
    """x fp32 [n, H, d] new rows, old scale fp32 [H] -> scale, inverse"""
    s = np.abs(x).max((0, 2)) * (F(1) / F(127))
    s = np.where(s < F(2.0 ** -96), F(0), s)
    s = np.where(np.isnan(s) | np.isnan(old), F("nan"), np.maximum(s, old)).astype(F)
    with np.errstate(divide="ignore"):
        return s, np.where(s > 0, F(1) / s, F(0)).astype(F)


def codes_of(x, inv):
    with np.errstate(invalid="ignore"):
        y = np.rint(x * inv[:, None])
    return np.clip(np.where(np.isnan(y), 0, y), -127, 127).astype(np.int64)


def store(cache, k, v, runs):
    """Writes into `cache` (a Cache), fp32 k, v [rows, H, d]."""
    for block, row, slot, n in runs:
        for which, x in enumerate((k, v)):
            x = x[row:row + n]
            old = cache.scales[block, :, which] if slot else np.zeros(x.shape[1], F)
            s, inv = quantize(x, old)
            codes = cache.codes[which][block]
            for i in range(slot):
                codes[i] = codes_of(codes[i].astype(F) * old[:, None], inv)
            for i in range(n):
                codes[slot + i] = codes_of(x[i], inv)
            codes[slot + n:] = 0
            cache.scales[block, :, which] = s


def attention(q, k, v):
    """q [N, Hq, d], k, v [n, H, d] in 64 bits -> out, and the largest sum of |q k| / sqrt(d)"""
    N, Hq, d = q.shape
    if len(k) == 0 or N == 0:
        return np.zeros_like(q), 0.0
    G = Hq // k.shape[1]
    out, big = np.zeros_like(q), 0.0
    for h in range(Hq):
        x = q[:, h] @ k[:, h // G].T / np.sqrt(d)
        big = max(big, float((np.abs(q[:, h]) @ np.abs(k[:, h // G]).T).max() / np.sqrt(d)))
        p = np.exp(x - x.max(1, keepdims=True))
        out[:, h] = p / p.sum(1, keepdims=True) @ v[:, h // G]
    return out, big


def tolerance(dtype, d, n, big, v, out, shift=16):
    """How far the kernel's output may be from attention()'s, from the roundings it makes (a bound, element by element).

    A logit: an fp32 query has 22 bits (2^-22), a 16-bit one all; d products summed in fp32 (d 2^-24), scaled and shifted
    (4 roundings): |dl| <= (2^-22 + (d + 4) 2^-24) sum |q k| / sqrt(d); log2 of a value's scale (|.| <= shift) adds its own
    roundings, 2 shift 2^-24.  exp turns it into a relative error, twice (a weight
    and the sum of all); 2^x and log2 of the hardware are good to 2^-22 each.  A weight rounds to 2^-22 (fp32) or 2^-11;
    weights below 2^-14 2^-6 of the largest to a multiple of 2^-24 2^-6, which n of them add.  The sums over n rows: n 2^-24
    each.  All of it times the largest |v|; then the output's own rounding."""
    u = 2.0 ** -22 if dtype == "fp32" else 2.0 ** -11
    logit = (2.0 ** -22 + (d + 4) * 2.0 ** -24) * big + 2 * shift * 2.0 ** -24
    rel = 2 * logit * 1.01 + 4 * 2.0 ** -22 + u + n * 2.0 ** -31 + 2 * (n + 40) * 2.0 ** -24
    half = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    least = {"fp32": 0.0, "fp16": 2.0 ** -25, "bf16": 0.0}[dtype]  # fp16's subnormal outputs
    return rel * np.abs(v).max() + half * np.abs(out) * 1.01 + least
