"""dgq_groupnorm in 64 bits, with the error that its kernels may make, from the roundings they take."""
import numpy as np

U = 2.0 ** -24
HALF_STEP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"fp32": 1e-35, "fp16": 2.0 ** -25, "bf16": 1e-35}  # where a type has no more bits; fp32: exponentials past 2^126


def groupnorm(x, starts, ends, groups, weight=None, bias=None, eps=1e-5, silu=False, add=None, scale=None, shift=None,
              out_type="fp32"):
    """x [rows, C], image b in rows starts[b] .. ends[b] - 1.  Returns (values, tolerance), NaN in rows of no image.

    The kernels hold x - p (p: fp32 next to the channel's mean), a = r w (1 + scale) and q in fp32, each rounded once, and
    t = (x - p) a + q rounded once: 2 U |x - p| |a| + U |q| + U |t|, of which twice as much is allowed for the 64-bit sums'
    part (tests keep means below 10^3 deviations: 10^6 2^-53 times the additions of a thread).  SiLU's slope is at most 1.1;
    2^x and 1 / x are good to 2 U, the exponent carries |t| U of its own and |t| U of its constant's."""
    x = x.astype(np.float64)
    rows, C = x.shape
    y, tol = np.full((rows, C), np.nan), np.full((rows, C), np.nan)
    one = np.ones(C)
    for b, (r0, r1) in enumerate(zip(starts, ends)):
        if r1 <= r0:
            continue
        v = x[r0:r1] + (0 if add is None else add[b].astype(np.float64))
        v = v.reshape(r1 - r0, groups, C // groups)
        mean = v.mean((0, 2), keepdims=True)
        r = 1 / np.sqrt(np.square(v - mean).mean((0, 2), keepdims=True) + eps)
        d = (v - mean).reshape(r1 - r0, C)
        r = np.broadcast_to(r, (1, groups, C // groups)).reshape(C)
        f = one if scale is None else 1 + scale[b].astype(np.float64)
        a = r * (one if weight is None else weight.astype(np.float64)) * f
        q = (0 * one if bias is None else bias.astype(np.float64)) * f + (0 if shift is None else shift[b].astype(np.float64))
        t = d * a + q
        off = 2 * U * (2 * np.abs(d * a) + np.abs(q) + np.abs(t))
        # p itself is rounded, which moves x - p and q against each other
        p = np.broadcast_to(mean, (1, groups, C // groups)).reshape(C) - (0 if add is None else add[b].astype(np.float64))
        off += 4 * U * U * np.abs(p) * np.abs(a)
        if silu:
            s = 1 / (1 + np.exp(-np.clip(t, -700, 700)))
            off = 1.1 * off + np.abs(t * s) * U * (6 + 2 * np.abs(t))
            t = t * s
        y[r0:r1] = t
        tol[r0:r1] = off + (np.abs(t) + off) * HALF_STEP[out_type] + TINY[out_type]
    return y, tol
