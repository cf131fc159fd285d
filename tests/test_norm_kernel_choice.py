"""The GPU tests of the group norm reach every kernel of it, of every type (on the CPU: the library's own choice for their sizes)."""
import ctypes

import pytest

import test_gpu_groupnorm as sizes

CHUNKS, TABLES = 0, 1
HOLD = [10, 11, 12, 13]  # 256 threads with 4 vectors, 1024 with 4, 8, 16


@pytest.fixture(scope="module")
def kernel():
    import os

    import paper_2501_04304_amd as dgq
    if not os.path.exists(dgq.LIB_PATH):
        from paper_2501_04304_amd import build
        build.build()
    f = dgq.lib().dgq_probe_groupnorm_kernel
    f.argtypes = [ctypes.c_int32, ctypes.c_int64] + [ctypes.c_int32] * 4
    return f


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_every_kernel(kernel, dtype):
    got = {s: kernel(s[0], s[1], 0, s[2], s[3], dtype) for s in sizes.SIZES + sizes.HELD}
    assert set(got.values()) == {CHUNKS, TABLES, *HOLD}, got


@pytest.mark.parametrize("dtype", [1, 2])
def test_packed_images_that_most_vectors_hold(kernel, dtype):
    front_and_behind = 5
    for lengths, C, G in sizes.HELD_PACKED:
        assert kernel(len(lengths), sum(lengths) + front_and_behind, 1, C, G, dtype) == HOLD[3], (lengths, C, G)


def test_what_is_not_a_call(kernel):
    for bad in ((0, 1, 0, 8, 1, 0), (1, 0, 0, 8, 1, 0), (1, 1, 0, 8, 3, 0), (1, 1, 0, 8, 1, 3), (1, 1, 0, 0, 1, 0)):
        assert kernel(*bad) == -1


def test_wide_launches(kernel):
    """2^24 groups of 256 threads, 2^22 of 1024: in chunks; one image fewer: held."""
    assert kernel(16384, 1, 0, 32768, 1024, 0) == CHUNKS and kernel(16383, 1, 0, 32768, 1024, 0) == 10
    assert kernel(4096, 129, 0, 32768, 1024, 0) in (CHUNKS, TABLES) and kernel(4095, 129, 0, 32768, 1024, 0) == 11
