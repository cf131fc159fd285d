"""The attention over the 8-bit cache at the ends of what logits and scales may be, at every kernel of it and both joins."""
import numpy as np
import pytest

from test_gpu_kv import _filled, _floats, _i32, _type, dgq  # noqa: F401  (dgq is a fixture)

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
