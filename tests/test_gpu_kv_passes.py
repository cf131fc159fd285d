"""The attention over short requests where a workgroup takes its rows in several passes: the request's tiles stay in LDS, the
next pass's queries are loaded under the present one, and queries and results change places in the same LDS."""
import numpy as np
import pytest

from test_gpu_kv import TYPES, _check_attention, _filled, _floats, _i32, dgq  # noqa: F401  (dgq is a fixture)

pytestmark = pytest.mark.gpu

# passes: S, H, G, d, queries of each request, lengths, columns.  No number of rows is a multiple of 32, or of a workgroup's.
EVEN = {
    2: (32, 32, 1, 24, 6100, [1, 77], 3),
    5: (32, 16, 3, 64, 10201, [100, 77], 4),
    16: (32, 64, 1, 8, 16300, [77, 0, 33], 3),
}
PACKED = (32, 40, 1, 40, [0, 1, 5000, 33, 127, 128, 129, 0, 4097, 300], [77, 3, 77, 0, 64, 33, 1, 5, 90, 32], 3)


def _check(held, table, lengths, qs, got, dtype, d, step):
    """Rows at both ends of every pass and workgroup against 64 bits; all rows against fp32 products, to what tells rows apart."""
    import torch
    rng = np.random.default_rng(1)
    some = []
    for q in qs:
        n = len(q)
        at = np.arange(0, n, 128)
        edges = (np.r_[at, np.arange(0, n, step), n][:, None] + np.arange(-2, 2)).ravel()
        edges = np.unique(edges[(edges >= 0) & (edges < n)])
        some.append(edges if len(edges) < 200 else np.unique(rng.choice(edges, 200)))
    _check_attention(held, table, lengths, [q[s] for q, s in zip(qs, some)], [x[s] for x, s in zip(got, some)], dtype, d)
    G = qs[0].shape[1] // held.codes[0].shape[2]
    for b, n in enumerate(lengths):
        if n == 0 or len(qs[b]) == 0:
            assert (got[b] == 0).all()
            continue
        k, v = (torch.from_numpy(held.exact(w, table, b, n).astype(np.float32)).cuda() for w in (0, 1))
        for h in range(qs[b].shape[1]):
            q = torch.from_numpy(np.ascontiguousarray(qs[b][:, h])).cuda()
            p = torch.softmax(q @ k[:, h // G].t().contiguous() / d ** 0.5, 1)
            far = (p @ v[:, h // G].contiguous() - torch.from_numpy(np.ascontiguousarray(got[b][:, h])).cuda()).abs().max()
            assert float(far) <= {"fp32": 1e-4, "fp16": 4e-3, "bf16": 2e-2}[dtype] * float(v.abs().max()), (b, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("passes", EVEN)
def test_passes(dgq, passes, dtype):  # noqa: F811
    import torch
    S, H, G, d, N, lengths, W = EVEN[passes]
    rng = np.random.default_rng(passes)
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=W)
    q, qn = _floats(rng, (len(lengths), N, H * G, d), dtype)
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths))
    again = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), out=torch.full_like(q, float("nan")))
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    _check(held, table, lengths, qn, out.float().cpu().numpy(), dtype, d, 128 * passes)


@pytest.mark.parametrize("dtype", TYPES)
def test_passes_of_packed_queries(dgq, dtype):  # noqa: F811
    import torch
    S, H, G, d, n, lengths, W = PACKED
    rng = np.random.default_rng(7)
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=W)
    starts = np.concatenate([[3], 3 + np.cumsum(n)])
    q, qn = _floats(rng, (starts[-1] + 5, H * G, d), dtype)
    out = torch.full_like(q, 7.0)
    dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), q_offsets=_i32(starts), out=out)
    on = out.float().cpu().numpy()
    assert (on[:3] == 7).all() and (on[starts[-1]:] == 7).all()
    at = [slice(*s) for s in zip(starts, starts[1:])]
    _check(held, table, lengths, [qn[s] for s in at], [on[s] for s in at], dtype, d, 256)
