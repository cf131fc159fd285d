"""Blocks of the 8-bit cache that several requests name, and rows that are coded again when their block grows."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import _cache, _check_attention, _floats, _i32, _read, dgq  # noqa: F401  (dgq is a fixture)

pytestmark = pytest.mark.gpu


def test_requests_that_share_full_blocks_grow_apart(dgq):  # noqa: F811
    """Three requests start from one prompt's two full blocks and get rows of their own, twice; a fourth reads what the first
    one has and gets none."""
    import torch
    rng = np.random.default_rng(30)
    S, H, d, B, W, n_blocks = 32, 2, 40, 4, 6, 20
    c = _cache(dgq, n_blocks, S, H, d)
    table = np.full((B, W), -1)
    free, d_free, d_n, d_table = list(rng.permutation(n_blocks)), None, _i32([n_blocks]), _i32(table)
    d_free = _i32(free)
    mirror = _read(c)
    lengths = [0] * B
    for step, new in enumerate(([64, 0, 0, 0], [9, 30, 70, 0], [40, 1, 0, 0])):
        if step == 1:  # the prompt's blocks to the others
            d_table[1:, :2] = d_table[0, :2]
            table[1:, :2] = table[0, :2]
            lengths = [64] * B
            shared = list(table[0, :2])
            before = {w: mirror.codes[w][shared].copy() for w in (0, 1)}
        rows = sum(new)
        plan = dgq.dgq_kv_plan(_i32(lengths), _i32(new), d_table, d_free, d_n, S, rows)
        table, lengths, n_free, _, runs, counts = ref.plan(lengths, new, table, free, len(free), S, rows)
        assert plan.counts.tolist() == counts and counts[2] == 0
        assert len({r[0] for r in runs}) == len(runs)  # no block twice
        free, d_n = free[:n_free], plan.n_free
        kv, kvn = _floats(rng, (rows, 2, H, d), "fp32")
        dgq.dgq_kv_store(c, kv[:, 0], kv[:, 1], plan.runs)
        ref.store(mirror, kvn[:, 0], kvn[:, 1], runs)
        q, qn = _floats(rng, (B, 7, H, d), "fp32")
        out = dgq.dgq_xattn_kv(q, c, d_table, plan.lengths)
        torch.cuda.synchronize()
        assert d_table.cpu().numpy().tolist() == table.tolist() and plan.lengths.tolist() == [int(n) for n in lengths]
        _check_attention(mirror, table, lengths, qn, out.cpu().numpy(), "fp32", d)
    got = _read(c)
    for w in (0, 1):
        assert np.array_equal(got.codes[w][shared], before[w])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_in_front_are_off_by_half_a_scale_for_every_growth(dgq, dtype):  # noqa: F811
    """Rows appended one by one, some larger than all before: a row is off by half of its first scale and half of every larger
    one since; where the scale stays, codes do."""
    import torch
    rng = np.random.default_rng(31)
    S, H, d = 64, 3, 24
    c = _cache(dgq, 2, S, H, d)
    size = np.cumprod(rng.choice([0.5, 1.0, 1.3, 1.9], S)).astype(np.float32)
    k, _ = _floats(rng, (S, H, d), "fp32")
    k = (k * torch.from_numpy(size).cuda()[:, None, None]).to(torch.float32 if dtype == "fp32" else torch.bfloat16)
    kn = k.float().cpu().numpy()
    off = np.zeros((S, H))
    last = None
    for r in range(S):
        dgq.dgq_kv_store(c, k, -k, _i32([(1, r, r, 1)]))
        torch.cuda.synchronize()
        got = _read(c)
        s = got.scales[1, :, 0].astype(np.float64)
        grown = s > last.scales[1, :, 0] if r else np.ones(H, bool)
        off[:r + 1] += np.where(grown, s * 0.5 * (1 + 2.0 ** -12), 0)  # (rounding next to a half: 127 steps of 3 2^-24)
        off[r] = s * 0.5 * (1 + 2.0 ** -12)
        for w, sign in ((0, 1), (1, -1)):
            x = got.codes[w][1, :r + 1] * got.scales[1, :, w].astype(np.float64)[:, None]
            assert (np.abs(x - sign * kn[:r + 1]).max(2) <= off[:r + 1]).all(), r
            if r:
                still = ~grown
                assert np.array_equal(got.codes[w][1, :r][:, still], last.codes[w][1, :r][:, still])
        last = got
