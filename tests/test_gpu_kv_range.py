"""The attention over the 8-bit cache at the ends of what logits and scales may be, at every kernel of it and both joins."""
import numpy as np
import pytest

from test_gpu_kv import TYPES, _filled, _floats, _i32, _type, dgq  # noqa: F401  (dgq is a fixture)

pytestmark = pytest.mark.gpu

FORMS = {  # S, H, d, queries of a request, rows of the longest request, columns of the table; three requests a call
    "few": (32, 2, 32, 5, 150, 6),
    "split": (32, 2, 32, 2, 2000, 64),          # four splits: joined by a wavefront a row
    "many splits": (64, 2, 64, 1, 20000, 314),  # forty: joined by a workgroup a row
    "short": (32, 2, 32, 5500, 200, 8),
    "stages": (32, 2, 32, 5500, 300, 11),
    "few, wide": (64, 2, 160, 5, 450, 8),       # one tile in registers
}
ENDS = {"fp32": 2.0 ** -20, "fp16": 2.0 ** -11 * 1.01, "bf16": 2.0 ** -8 * 1.01}
# a row that has all the weight: 2^6 in fp16 pieces, the reciprocal of the scale and the division (2^-22 each at most), then
# the output's own half step


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("form", FORMS)
def test_logits_far_below_zero(dgq, form, dtype):  # noqa: F811
    """All of a request's logits between -1e33 and -1e35: the largest takes all the weight, also where it is the only one."""
    S, H, d, N, rows, W = FORMS[form]
    rng = np.random.default_rng(rows + N)
    lengths, best = [1, 2, rows], [0, 1, rows - 7]
    at = [b + sum(lengths[:i]) for i, b in enumerate(best)]

    def gain(k, v):
        k.fill_(-3)
        k[at] = -2
        return k, v
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=W, gain=gain)
    q, _ = _floats(rng, (3, N, H, d), "fp32")
    q = (q.abs() + 1).mul(3e32).to(_type(dtype))
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths)).float().cpu().numpy()
    for b, r in enumerate(best):
        want = held.values(1, table[b, r // S], r % S)
        assert (np.abs(out[b] - want) <= ENDS[dtype] * np.abs(want)).all(), (b, out[b, 0, 0, :4], want[0, :4])


def _of_a_billion(dgq, form, dtype, zeros):  # noqa: F811
    S, H, d, N, rows, W = FORMS[form]
    rng = np.random.default_rng(rows + N + 1)
    lengths = [60, rows // 2, rows]

    def gain(k, v):
        if zeros:  # every third block of every request
            at = np.concatenate([np.arange(n) // S % 3 == 1 for n in lengths])
            v[at] = 0
        return k * 3e4, v
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=W, gain=gain)
    q, _ = _floats(rng, (3, N, H, d), "fp32")
    q = (q * 1e4).clamp(-65504, 65504).to(_type(dtype))
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths)).float().cpu().numpy()
    qn = q.double().cpu().numpy()
    seen = 0
    for b, n in enumerate(lengths):
        k, v = (held.exact(w, table, b, n) for w in (0, 1))
        for h in range(H):
            some = np.arange(N) if N < 600 else rng.choice(N, 600, replace=False)
            x = qn[b, some, h] @ k[:, h].T / np.sqrt(d)
            big = (np.abs(qn[b, some, h]) @ np.abs(k[:, h]).T).max(1) / np.sqrt(d)
            order = np.argsort(x, 1)
            first, second = order[:, -1], order[:, -2]
            rows_ = np.arange(len(some))
            # clear of the logits' roundings, (2^-22 + (d + 8) 2^-24) of sum |q k| each: the largest takes all
            clear = x[rows_, first] - x[rows_, second] > 4 * (2.0 ** -22 + (d + 8) * 2.0 ** -24) * big + 1000
            want = v[first[clear], h]
            err = np.abs(out[b, some[clear], h] - want)
            assert (err <= ENDS[dtype] * np.abs(want)).all(), (b, h, float(np.nanmax(err)), int((~(err <= ENDS[dtype] * np.abs(want))).any(1).sum()))
            seen += int(clear.sum())
    assert seen >= 0.8 * min(N, 600) * 3 * H


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_logits_of_a_billion(dgq, form, dtype):  # noqa: F811
    """Logits whose neighbours in fp32 lie 16 to 1024 apart: the running maximum has to be the very number that the largest
    row's logit is, next to which the row's weight is 1."""
    _of_a_billion(dgq, form, dtype, zeros=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_zero_values_beside_logits_of_a_billion(dgq, form, dtype):  # noqa: F811
    """The same where every third block's values are zeros: its rows take weight, or leave it, like any others."""
    _of_a_billion(dgq, form, dtype, zeros=True)


@pytest.mark.parametrize("dtype,small,large", [("fp32", -90, 45), ("fp32", -95, 9), ("fp32", -95, 118), ("bf16", -90, 45),
                                               ("bf16", -95, 9), ("bf16", -95, 118), ("fp16", -95, 9)])  # fp16 holds no larger mean
@pytest.mark.parametrize("last", [False, True], ids=["large_first", "small_first"])
@pytest.mark.parametrize("form", FORMS)
def test_equal_logits_over_scales_far_apart(dgq, form, last, dtype, small, large):  # noqa: F811
    """Rows of equal weight in blocks of values near 2^small, near 2^large and of zeros: the mean of all, however many times
    one scale is the other.  (A tile, a wavefront's share and a split each meet both.)"""
    S, H, d, N, rows, W = FORMS[form]
    rng = np.random.default_rng(rows + N + 2)
    lengths = [S + 20, rows // 2, rows]

    def gain(k, v):
        at = np.concatenate([np.arange(n) // S for n in lengths])
        one = np.concatenate([(np.arange(n) // S < -(-n // S) // 2) == last for n in lengths])  # halves, at either end
        f = np.where(one, 2.0 ** small, 2.0 ** large) * np.where(at % 5 == 3, 0, 1)
        import torch
        v = v.abs().clamp(0.5, 4) * torch.from_numpy(f.astype(np.float32)).cuda()[:, None, None]
        k.zero_()
        return k, v
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=W, gain=gain)
    q, _ = _floats(rng, (3, N, H, d), dtype)
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths)).float().cpu().numpy()
    for b, n in enumerate(lengths):
        want = held.exact(1, table, b, n).mean(0)  # all values positive: nothing cancels
        # a weight in fp16 pieces (2^-22, 2^-11), 2^x and 1/x of the hardware (2^-22 each, twice), n sums in fp32
        rel = (2.0 ** -22 if dtype == "fp32" else 2.0 ** -11) + 4 * 2.0 ** -22 + 2 * (n + 40) * 2.0 ** -24
        lim = (rel + {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype] * 1.01) * want
        assert (np.abs(out[b] - want) <= lim).all(), (b, float((out[b] / want).min()), float((out[b] / want).max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_softmax_over_scales_far_apart(dgq, form, dtype):  # noqa: F811
    """Values that grow and shrink from block to block, by 2^40 or what the type holds, among them blocks of zeros; the weight
    lies on a few rows of any of them.  Each element is held to its own sum of p |v|, so that a wrong denominator shows."""
    import torch
    S, H, d, N, rows, W = FORMS[form]
    rng = np.random.default_rng(rows + N + 3)
    lengths = [S + 9, rows // 2, rows]

    def gain(k, v):
        f = []
        for n in lengths:
            e = 2.0 ** rng.integers(-40, 9 if dtype == "fp16" else 41, -(-n // S))
            e[3::4] = 0
            f.append(np.repeat(e, S)[:n])
        return k * 3, v * torch.from_numpy(np.concatenate(f).astype(np.float32)).cuda()[:, None, None]
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=W, gain=gain)
    q, _ = _floats(rng, (3, N, H, d), dtype)
    q = q * 4
    qn = q.float().cpu().numpy()
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths)).float().cpu().numpy()
    told = seen = 0
    for b, n in enumerate(lengths):
        k, v = (held.exact(w, table, b, n) for w in (0, 1))
        s = np.stack([held.scales[table[b, r // S], :, 1] for r in range(n)]).astype(np.float64)
        some = np.arange(N) if N < 200 else rng.choice(N, 200, replace=False)
        for h in range(H):
            x = qn[b, some, h].astype(np.float64) @ k[:, h].T / np.sqrt(d)
            big = float((np.abs(qn[b, some, h]) @ np.abs(k[:, h]).T).max() / np.sqrt(d))
            p = np.exp(x - x.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            want = p @ v[:, h]
            # A logit: kv_reference.tolerance's.  A weight: 2^-22 or 2^-11, 2^x, log2 and 1/x 2^-22 each; one that is below fp16's normals
            # is off by 2^-25 2^-6 of the largest (in units of what a row adds), and where the line below is the sum of such
            # weights, of scales at most 2^6 apart, by 2^6 times as much.  The sums: 2 (n + 40) 2^-24.
            logit = (2.0 ** -22 + (d + 4) * 2.0 ** -24) * big + 2 * 64 * 2.0 ** -24
            rel = 2 * logit * 1.01 + 6 * 2.0 ** -22 + 2 * (n + 40) * 2.0 ** -24
            rel += 2.0 ** -22 if dtype == "fp32" else 2.0 ** -11 + n * 2.0 ** -25
            lim = rel * (p @ np.abs(v[:, h])) + n * 2.0 ** -31 * 127 * (p * s[:, h]).max(1)[:, None]
            lim += {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype] * 1.01 * np.abs(want)
            if dtype == "fp16":
                lim += 2.0 ** -25  # its subnormal numbers
            assert (np.abs(out[b, some, h] - want) <= lim).all(), (b, h, float((np.abs(out[b, some, h] - want) / lim).max()))
            told += int((lim.max(1) < 0.5 * np.abs(want).max(1)).sum())
            seen += len(some)
    assert told >= (0.6 if dtype == "fp16" else 0.9) * seen  # rows where zeros, or twice the output, would not pass
