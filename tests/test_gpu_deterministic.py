"""New tensors under torch.use_deterministic_algorithms: torch fills what it hands out, so that rows which a call leaves as they
were hold NaN and not whatever the allocator had there, and the fill stands in front of the call's own work on its stream."""
import numpy as np
import pytest

import dgq_inputs as di

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dgq():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_04304_amd as m
    m.lib()
    return m


@pytest.fixture
def deterministic():
    import torch
    before = torch.are_deterministic_algorithms_enabled(), torch.is_deterministic_algorithms_warn_only_enabled()
    assert torch.utils.deterministic.fill_uninitialized_memory
    torch.use_deterministic_algorithms(True, warn_only=True)
    yield
    torch.use_deterministic_algorithms(before[0], warn_only=before[1])


def _i32(v):
    import torch
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _sevens(nbytes):
    """Memory that the allocator hands out next, full of sevens."""
    import torch
    torch.full((nbytes // 4,), 7.0, device="cuda")
    torch.cuda.synchronize()


@pytest.mark.parametrize("lengths", [[40, 0, 3], [9000, 1]])  # held by workgroups, and in chunks
def test_groupnorm(dgq, deterministic, lengths):
    import torch
    C, G, front, behind = 64, 4, 3, 2
    offsets = front + np.concatenate([[0], np.cumsum(lengths)])
    rows = int(offsets[-1]) + behind
    x = torch.randn((rows, C), device="cuda")
    _sevens(rows * C * 4)
    out = dgq.dgq_groupnorm(x, G, offsets=_i32(offsets))
    assert torch.isnan(out[:front]).all() and torch.isnan(out[rows - behind:]).all()
    assert not torch.isnan(out[front:rows - behind]).any()


def test_attention_over_the_cache(dgq, deterministic):
    import torch
    S, H, d, front, behind = 32, 2, 64, 4, 5
    c = dgq.KVCache.empty(4, S, H, d)
    k = torch.randn((S, H, d), device="cuda")
    dgq.dgq_kv_store(c, k, k, _i32([[1, 0, 0, S]]))
    q = torch.randn((front + 10 + behind, H, d), device="cuda")
    _sevens(q.numel() * 4)
    out = dgq.dgq_xattn_kv(q, c, _i32([[1]]), _i32([S]), q_offsets=_i32([front, front + 10]))
    assert torch.isnan(out[:front]).all() and torch.isnan(out[-behind:]).all()
    assert not torch.isnan(out[front:-behind]).any()


def test_the_fill_is_in_front_of_a_call_on_another_stream(dgq, deterministic):
    """The current stream is kept busy, so that a fill there would come behind the call's own writes."""
    import torch
    run, cal = di.linear_case(7, 2, 128, 320, 192), di.linear_case(7, 2, 128, 320, 192, calib=True)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    g = dgq.dgq_calibrate_groups(up(cal["X"]), 8, 64, 2)
    w = dgq.dgq_pack_weight(g, up(run["W"]), None, 8)
    x = up(run["X"])
    codes, cls = dgq.dgq_quantize_act(g, x)
    y = dgq.dgq_linear(g, w, codes, cls)
    n = dgq.dgq_groupnorm(x.view(2, 128, 320), 32)
    side, busy = torch.cuda.Stream(), torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-3
    codes2, cls2 = dgq.dgq_quantize_act(g, x, stream=side)
    y2 = dgq.dgq_linear(g, w, codes2, cls2, stream=side)
    n2 = dgq.dgq_groupnorm(x.view(2, 128, 320), 32, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(codes, codes2) and torch.equal(cls, cls2) and torch.equal(y, y2) and torch.equal(n, n2)
