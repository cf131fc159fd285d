"""Rows that are split over the chip and joined: every split has to arrive.  (A mean over thousands of random rows is so near
zero that a bound on its roundings says little about any one split.)"""
import numpy as np
import pytest

from test_gpu_kv import TYPES, _filled, _i32, _type, dgq  # noqa: F401  (dgq is a fixture)
from test_gpu_kv_range import ENDS

pytestmark = pytest.mark.gpu

LEAST = 512  # rows: the shortest split of a long request
SHAPES = [  # d, rows, splits (one wave's queries: nothing longer than LEAST)
    (8, 140000, 274), (64, 20000, 40), (256, 6000, 12), (128, 7000, 14), (40, 8100, 16), (256, 4000, 8), (160, 9000, 18), (24, 520, 2)]


def _directions(d, n, rng):
    """n distinct vertices of a cube, +-1"""
    if d == 8:
        return (rng.permutation(256)[:n, None] >> np.arange(8) & 1) * 2.0 - 1
    x = rng.choice([-1.0, 1.0], (n, d))
    assert len(np.unique(x, axis=0)) == n
    return x


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rows,splits", SHAPES)
def test_every_split_may_hold_the_row(dgq, d, rows, splits, dtype, packed):  # noqa: F811
    """A query that one row answers, for a row of each split (of d = 8, of 256 splits at both ends): the output is that row."""
    import torch
    rng = np.random.default_rng(d + rows)
    S, G, N = 64, 3, 4
    at = np.array([min(s * LEAST + int(rng.integers(LEAST)), rows - 1) for s in range(-(-rows // LEAST))])
    if len(at) > 256:
        at = np.r_[at[:128], at[-128:]]
    way = _directions(d, len(at), rng)
    size = (20 * d ** 0.5) ** 0.5  # the next vertex differs in one dim, and its logit by 2 size^2 / sqrt(d) = 40

    def gain(k, v):
        k.zero_()
        k[torch.from_numpy(at).cuda(), 0] = torch.from_numpy((way * size).astype(np.float32)).cuda()
        return k, v
    c, table, held = _filled(dgq, rng, [rows], S, 1, d, gain=gain)
    t, n = _i32(table), _i32([rows])
    per = d * 4 + 8
    assert dgq.dgq_xattn_kv_workspace_bytes(1, N, packed, G, 1, d, table.shape[1], S) == splits * N * G * per
    for i in range(0, len(at), N * G):
        aim = np.resize(np.arange(i, min(i + N * G, len(at))), N * G)
        q = torch.from_numpy((way[aim] * size).astype(np.float32)).cuda().to(_type(dtype)).view(1, N, G, d)
        if packed:
            out = dgq.dgq_xattn_kv(q[0], c, t, n, q_offsets=_i32([0, N]))
        else:
            out = dgq.dgq_xattn_kv(q, c, t, n)
        got = out.float().cpu().numpy().reshape(N * G, d)
        want = np.stack([held.values(1, table[0, r // S], r % S)[0] for r in at[aim]])
        # e^-40 of every other row
        lim = ENDS[dtype] * np.abs(want) + rows * np.exp(-39) * 4
        assert (lim.max(1) < 0.02 * np.abs(want).max(1)).all()  # zeros, or another row, would show
        assert (np.abs(got - want) <= lim).all(), (i, float((np.abs(got - want) / lim).max()))


@pytest.mark.parametrize("d,rows,splits", SHAPES)
def test_mean_of_all_splits(dgq, d, rows, splits):  # noqa: F811
    """Equal logits over values of one sign, those of every other split three times the rest's: a split too few, or a part of
    one, moves the mean by far more than the sums' roundings."""
    import torch
    rng = np.random.default_rng(d + rows + 1)
    S, N = 64, 2

    def gain(k, v):
        k.zero_()
        f = torch.from_numpy(np.where(np.arange(rows) // LEAST % 2, 3.0, 1.0).astype(np.float32)).cuda()
        return k, (1 + 0.1 * v.clamp(-3, 3)) * f[:, None, None]
    c, table, held = _filled(dgq, rng, [rows], S, 1, d, gain=gain)
    q = torch.randn(1, N, 1, d, device="cuda")
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32([rows])).cpu().numpy()
    want = held.exact(1, table, 0, rows).mean(0)
    # A wavefront adds up at most 4 tiles of 32 rows, four of them meet, and a join adds up to 3 splits to a thread and 128 threads:
    # fewer than 300 sums of one sign, above and below the line.  A weight: 2^-22 in its pieces, 2^x and 1/x 2^-22 each, two roots.
    rel = 2 * 300 * 2.0 ** -24 + 6 * 2.0 ** -22
    assert rel * 20 < 0.25 / splits  # what the least split moves, were it full
    assert (np.abs(out[0] - want) <= rel * want).all(), float(np.abs(out[0] / want - 1).max())
