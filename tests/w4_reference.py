"""Weights in 4 bits, by their definition, in numpy."""
import numpy as np

NAN_WORD = 0x7FC00000


def quantize(w, group):
    """fp32 [O, C] -> codes int64 [16 R, 128 T], words uint32 [16 R, 128 T / group]; every operation in fp32."""
    O, C = w.shape
    full = np.zeros((-(-O // 16) * 16, -(-C // 128) * 128), np.float32)
    full[:O, :C] = w
    w = full.reshape(len(full), -1, group)
    with np.errstate(all="ignore"):
        lo, hi = np.minimum(np.fmin.reduce(w, 2), 0), np.maximum(np.fmax.reduce(w, 2), 0)
        spread = hi - lo
        bad = ~np.isfinite(w).all(2) | ~np.isfinite(spread)
        s = ((spread * np.float32(1 / 15)).view(np.uint32) & np.uint32(0xFFFFFFF0)).view(np.float32)
        s = np.where(s >= np.float32(2.0 ** -96), s, np.float32(0))
        inv = np.where(s > 0, np.float32(1) / s, np.float32(0))
        zero = np.clip(np.rint(-lo * inv), 0, 15)
        code = np.clip(np.rint(w * inv[:, :, None]) + zero[:, :, None], 0, 15)
    code[bad], zero[bad] = 0, 0
    words = s.view(np.uint32) | zero.astype(np.uint32)
    words[bad] = NAN_WORD
    return code.astype(np.int64).reshape(len(full), -1), words


def lay_out(codes, words, group):
    """The bytes of dgq_w4_bytes."""
    rows, C = codes.shape
    R, T = rows // 16, C // 128
    out = np.zeros((R, T, 4, 16, 4), np.uint32)  # q, r, j
    for k in range(128):
        j, q, i = k // 32, k // 8 % 4, k % 8
        part = codes[:, k::128].reshape(R, 16, T).transpose(0, 2, 1).astype(np.uint32)
        out[:, :, q, :, j] |= part << np.uint32(4 * (i // 2 if i % 2 == 0 else 4 + i // 2))
    w = words.reshape(R, 16, T, 128 // group).transpose(0, 2, 1, 3)
    return np.concatenate([out.reshape(-1), np.ascontiguousarray(w).reshape(-1)]).view(np.uint8)


def values(codes, words, group, O, C):
    """fp64 [O, C]"""
    s = (words & np.uint32(0xFFFFFFF0)).view(np.float32).astype(np.float64)
    zero = (words & 15).astype(np.int64)
    v = (codes.reshape(len(codes), -1, group) - zero[:, :, None]) * s[:, :, None]
    return v.reshape(len(codes), -1)[:O, :C]


def silu(t):
    return t / (1 + np.exp(-np.clip(t, -700, 700)))


def matvec(x, codes, words, group, O, bias=None, act=False, out_type="fp32", pieces=1):
    """(y, tolerance) [M, O].

    A group's sum of x (code - zero) has at most group * pieces additions whose parts are at most sum |x| |code - zero| (a step
    each, 2^-23, for cores that cut); fp32 rows are held to 2^-23; scale and power come in one rounding each, and the groups'
    sums one each.  Elements far below their unit's largest add 2^-39 of that.  Then 16 v + bias, SiLU (norm_reference) and the
    type."""
    from norm_reference import HALF_STEP, TINY, U
    M, C = x.shape
    x = x.astype(np.float64)
    v = values(codes, words, group, O, C)
    y = x @ v.T
    n = -(-C // group)
    part = np.abs(x) @ np.abs(v).T
    unit = np.zeros((M, -(-C // 128) * 128))
    unit[:, :C] = np.abs(x)
    top = np.repeat(unit.reshape(M, -1, 128).max(2), 128, axis=1)[:, :C]
    off = part * U * (2 * min(group, C) * pieces + 2 + n + 4) + 2.0 ** -39 * top @ np.abs(v).T
    if bias is not None:
        y = y + bias.astype(np.float64)
    off = off + U * np.abs(y)
    if act:
        off = 1.1 * off + np.abs(silu(y)) * U * (6 + 2 * np.abs(y))
        y = silu(y)
    return y, off + (np.abs(y) + off) * HALF_STEP[out_type] + TINY[out_type]
