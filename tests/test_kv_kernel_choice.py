"""The GPU tests of the attention over the 8-bit cache reach every kernel of it, at several head widths (on the CPU: the
library's own choice for their shapes)."""
import ctypes

import pytest

import test_gpu_kv

FEW, SPLIT, SHORT, STAGES = 0, 1, 2, 3


@pytest.fixture(scope="module")
def kernel():
    import os

    import paper_2501_04304_amd as dgq
    if not os.path.exists(dgq.LIB_PATH):
        from paper_2501_04304_amd import build
        build.build()
    f = dgq.lib().dgq_probe_xattn_kv_kernel
    f.argtypes = [ctypes.c_int32, ctypes.c_int64] + [ctypes.c_int32] * 6
    return f


def _of(kernel, shape, width=None):
    S, H, G, d, N, lengths = shape
    return kernel(len(lengths), N, 0, H * G, H, d, width or -(-max(lengths) // S) + 1, S)


def test_few_rows(kernel):
    got = {s[:5]: _of(kernel, s) for s in test_gpu_kv.SHAPES}
    assert set(got.values()) == {FEW, SPLIT}, got
    assert len({s[3] // 64 for s in test_gpu_kv.SHAPES}) >= 4


def test_many_rows(kernel):
    got = {s[:5]: _of(kernel, s, test_gpu_kv.width_of(s[0], s[5])) for s in test_gpu_kv.MANY}
    assert set(got.values()) == {SHORT, STAGES}, got
    for which in (SHORT, STAGES):
        widths = {-(-s[3] // 32) for s in got if got[s] == which}
        assert len(widths) >= 7, (which, widths)


def test_what_is_no_call(kernel):
    for bad in ((0, 1, 0, 1, 1, 8, 1, 32), (1, 0, 0, 1, 1, 8, 1, 32), (1, 1, 0, 3, 2, 8, 1, 32), (1, 1, 0, 1, 1, 8, 0, 32)):
        assert kernel(*bad) == -1
