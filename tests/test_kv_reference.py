"""The tests' plain forms of the 8-bit cache (kv_reference), and the calls' refusals, without a GPU."""
import ctypes as C

import numpy as np
import pytest

import kv_reference as ref


@pytest.fixture(scope="module")
def lib():
    import os

    import paper_2501_04304_amd as dgq
    if not os.path.exists(dgq.LIB_PATH):
        from paper_2501_04304_amd import build
        build.build()
    return dgq.lib()


def test_places_are_a_permutation():
    assert sorted(sum(ref.places(), [])) == list(range(32))


def test_plan_by_hand():
    table = np.full((3, 4), -1)
    got = ref.plan([30, 0, 64], [5, 40, 1], table, [10, 11, 12, 13, 14], 5, 32, 46)
    assert got[0].tolist() == [[-1, 14, -1, -1], [13, 12, -1, -1], [-1, -1, 11, -1]]
    assert got[1] == [35, 40, 65] and got[2] == 1 and got[3] == [0, 5, 45, 46]
    assert got[4] == [(-1, 0, 30, 2), (14, 2, 0, 3), (13, 5, 0, 32), (12, 37, 0, 8), (11, 45, 0, 1)]
    assert got[5] == [5, 4, 0, 46]


def test_store_and_attention_by_hand():
    """Two rows of one head: the codes of the largest are +-127, and the attention is the softmax's."""
    S, d = 32, 8
    c = ref.Cache(np.full(S * 2 * 16 + 8, 128, np.uint8), 1, S, 1, d)
    x = np.zeros((2, 1, d), np.float32)
    x[0, 0, 0], x[1, 0, 1] = 2.54, -1.27
    ref.store(c, x, 2 * x, [(0, 0, 0, 2)])
    assert c.codes[0][0, 0, 0, 0] == 127 and c.codes[0][0, 1, 0, 1] == -64
    assert np.allclose(c.scales[0, 0], [0.02, 0.04])
    out, _ = ref.attention(np.ones((1, 1, d)), c.exact(0, np.array([[0]]), 0, 2), c.exact(1, np.array([[0]]), 0, 2))
    p = np.exp(np.array([2.54, -1.28]) / np.sqrt(8))
    assert np.allclose(out[0, 0, :2], p / p.sum() * [5.08, -2.56], atol=1e-6)


def test_cache_bytes(lib):
    size = lib.dgq_kv_cache_bytes
    assert size(3, 32, 2, 40) == 3 * 2 * (32 * 2 * 48 + 8)
    assert size(1 << 20, 128, 16, 256) == (1 << 20) * 16 * (128 * 512 + 8)
    for bad in ((0, 32, 2, 40), (3, 48, 2, 40), (3, 32, 0, 40), (3, 32, 2, 20), (3, 32, 2, 264), (3, 32, 2, 0), (3, 32, 1 << 16, 8)):
        assert size(*bad) == 0


def test_refusals(lib):
    """Every argument that the calls name, before anything is enqueued."""
    buf = C.create_string_buffer(4096)
    p = (C.addressof(buf) + 15) // 16 * 16
    o, q = p + 64, p + 8  # another aligned buffer, a misaligned one

    def plan(code, **kw):
        a = dict(lengths=p, new=p, B=2, S=32, rows=10, table=p, W=4, free=p, cap=8, n=p, l2=o, n2=o, offs=p, runs=p, most=4, counts=p)
        a.update(kw)
        assert lib.dgq_kv_plan(*a.values(), None) == code, kw
    for name in ("lengths", "new", "table", "free", "n", "l2", "n2", "offs", "runs", "counts"):
        plan(-1, **{name: None})
    plan(-4, S=16), plan(-4, S=0), plan(-1, B=0), plan(-1, W=0), plan(-4, B=4097, most=9000), plan(-4, W=1 << 27)
    plan(-1, rows=-1), plan(-1, cap=0), plan(-4, rows=1 << 31, most=1 << 30), plan(-1, l2=p), plan(-1, n2=p), plan(-3, most=3)
    plan(-2, runs=q), plan(-2, counts=q)

    def release(code, **kw):
        a = dict(done=p, lengths=p, table=p, B=2, W=4, S=32, free=p, cap=8, n=p, l2=o, n2=o)
        a.update(kw)
        assert lib.dgq_kv_release(*a.values(), None) == code, kw
    for name in ("done", "lengths", "table", "free", "n", "l2", "n2"):
        release(-1, **{name: None})
    release(-4, S=33), release(-1, B=0), release(-4, B=4097), release(-1, cap=0), release(-1, l2=p), release(-1, n2=p)

    def store(code, **kw):
        a = dict(k=p, v=p, dtype=0, rows=4, kr=16, kh=16, vr=16, vh=16, runs=p, n=1, cache=p, blocks=1, S=32, H=1, d=16)
        a.update(kw)
        assert lib.dgq_kv_store(*a.values(), None) == code, kw
    for name in ("k", "v", "runs", "cache"):
        store(-1, **{name: None})
    for name in ("k", "v", "runs", "cache"):
        store(-2, **{name: q})
    for name in ("kr", "kh", "vr", "vh"):
        store(-2, **{name: 18}), store(-2, **{name: -16}), store(-2, **{name: 20, "dtype": 1})
    store(-1, dtype=3), store(-1, rows=-1), store(-1, n=-1), store(-4, rows=1 << 31), store(-4, n=1 << 24)
    store(-1, blocks=0), store(-1, H=0), store(-4, S=256), store(-4, d=12), store(-4, d=264), store(-4, H=65536)
    store(0, rows=0), store(0, n=0)  # nothing to write

    def load(code, **kw):
        a = dict(cache=p, blocks=1, S=32, H=1, d=16, table=p, W=1, lengths=p, B=1, rows=4, dtype=0, k=p, v=p)
        a.update(kw)
        assert lib.dgq_kv_load(*a.values(), None) == code, kw
    for name in ("cache", "table", "lengths", "k", "v"):
        load(-1, **{name: None})
    load(-2, cache=q), load(-2, k=q), load(-2, v=q), load(-1, dtype=-1), load(-1, rows=-1), load(-1, B=0), load(-4, B=65536)
    load(-4, rows=1 << 29)
    load(-4, d=20), load(-1, W=0), load(0, rows=0)

    def attend(code, **kw):
        a = dict(q=p, dtype=0, offsets=None, sb=64, sn=16, sh=16, B=1, N=64, Hq=2, cache=p, blocks=1, S=32, H=1, d=16, table=p, W=1,
                 lengths=p, out=p, ws=None, nbytes=0)
        a.update(kw)
        assert lib.dgq_xattn_kv(*a.values(), None) == code, kw
    for name in ("q", "cache", "table", "lengths", "out"):
        attend(-1, **{name: None})
    for name in ("q", "cache", "out"):
        attend(-2, **{name: q})
    for name in ("sb", "sn", "sh"):
        attend(-2, **{name: 2}), attend(-2, **{name: -4}), attend(-2, **{name: 4, "dtype": 2})
    attend(-1, dtype=4), attend(-1, N=-1), attend(-1, Hq=0), attend(-4, Hq=3, H=2), attend(-4, d=4), attend(-4, S=8), attend(-1, B=0)
    attend(-4, N=1 << 31), attend(-4, N=1 << 30, Hq=4), attend(-4, W=1 << 26), attend(0, N=0)
    attend(-4, N=1, B=1 << 20, H=32, Hq=32), attend(-4, N=1, B=1 << 20, W=1 << 14, H=2, ws=p, nbytes=1 << 60)
    need = lib.dgq_xattn_kv_workspace_bytes(1, 1, 0, 2, 1, 16, 64, 32)
    assert need > 0
    attend(-6, N=1, W=64, ws=None), attend(-6, N=1, W=64, ws=p, nbytes=need - 1), attend(-6, N=1, W=64, ws=q, nbytes=need)
    assert lib.dgq_xattn_kv_workspace_bytes(1, 64, 0, 3, 2, 16, 64, 32) == 0
    assert b"dgq_xattn_kv" in lib.dgq_last_error()
