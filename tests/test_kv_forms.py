"""The shapes of the tests reach the kernels, joins and passes that they are named for (on the CPU: the library's own choice)."""
import ctypes

import test_gpu_kv_passes
import test_gpu_kv_range as gpu
import test_gpu_kv_splits
from test_kv_kernel_choice import FEW, SHORT, SPLIT, STAGES, kernel  # noqa: F401  (kernel is a fixture)

import paper_2501_04304_amd as dgq


def test_forms(kernel):  # noqa: F811
    want = {"few": FEW, "split": SPLIT, "many splits": SPLIT, "short": SHORT, "stages": STAGES, "few, wide": FEW}
    for name, (S, H, d, N, rows, W) in gpu.FORMS.items():
        assert rows <= W * S
        assert kernel(3, N, 0, H, H, d, W, S) == want[name], name
        row = 3 * N * H * (d + 2) * 4
        splits = dgq.dgq_xattn_kv_workspace_bytes(3, N, False, H, H, d, W, S) // row
        if name == "split":
            assert 2 <= splits <= 16 and splits * d <= 2048
        elif name == "many splits":
            assert splits > 16
        else:
            assert splits == 0


def test_passes():
    rows = dgq.lib().dgq_probe_xattn_kv_rows
    rows.argtypes = [ctypes.c_int32, ctypes.c_int64] + [ctypes.c_int32] * 6
    for passes, (S, H, G, d, N, lengths, W) in test_gpu_kv_passes.EVEN.items():
        assert max(lengths) <= W * S and N * G % 32 and N * G % 128 and N * G > 128 * passes
        assert rows(len(lengths), N, 0, H * G, H, d, W, S) == 128 * passes
    S, H, G, d, n, lengths, W = test_gpu_kv_passes.PACKED
    assert rows(len(n), sum(n) + 8, 1, H * G, H, d, W, S) == 256
    assert rows(0, 1, 0, 1, 1, 8, 1, 32) == -1


def test_passes_take_the_kernel_of_short_requests(kernel):  # noqa: F811
    for S, H, G, d, N, lengths, W in test_gpu_kv_passes.EVEN.values():
        assert kernel(len(lengths), N, 0, H * G, H, d, W, S) == SHORT
    S, H, G, d, n, lengths, W = test_gpu_kv_passes.PACKED
    assert kernel(len(n), sum(n) + 8, 1, H * G, H, d, W, S) == SHORT


def test_splits():
    """of two queries and of four, with a head or three of them to the cached one"""
    joins = set()
    for d, rows, splits in test_gpu_kv_splits.SHAPES:
        width = -(-rows // 64) + 1
        for N, Hq in ((4, 3), (2, 1)):
            for packed in (False, True):
                assert dgq.dgq_xattn_kv_workspace_bytes(1, N, packed, Hq, 1, d, width, 64) == splits * N * Hq * (d + 2) * 4, d
        joins.add("one pass" if 16 < splits <= 256 else "two" if splits > 256 else "a wavefront" if splits * d <= 2048 else "one pass")
    assert joins == {"one pass", "two", "a wavefront"}
