"""Group norm and 4-bit weights: refusals of the C calls, and their sizes, without a GPU."""
import ctypes as C
import os

import numpy as np
import pytest

import norm_reference
import w4_reference


@pytest.fixture(scope="module")
def lib():
    import paper_2501_04304_amd as dgq
    if not os.path.exists(dgq.LIB_PATH):
        from paper_2501_04304_amd import build
        build.build()
    return dgq.lib()


BUF = (C.c_float * 256)()
P = (C.addressof(BUF) + 15) & ~15
EINVAL, EALIGN, EUNSUPPORTED, EWORKSPACE = -1, -2, -4, -6


def _norm(lib, **kw):
    a = dict(x=P, dtype=0, batch=64, row=8, offsets=None, B=1, N=8, C=8, G=2, weight=None, bias=None, eps=1e-5, add=None, add_s=0,
             scale=None, scale_s=0, shift=None, shift_s=0, act=0, out=P, out_dtype=0, ws=None, ws_bytes=0, stream=None)
    a.update(kw)
    return lib.dgq_groupnorm(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(dtype=3), EINVAL), (dict(dtype=1, out_dtype=2), EINVAL),
    (dict(dtype=0, out_dtype=1), EINVAL), (dict(act=2), EINVAL), (dict(act=-1), EINVAL), (dict(eps=-1e-9), EINVAL),
    (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(B=0), EINVAL), (dict(N=-1), EINVAL), (dict(C=0), EINVAL),
    (dict(G=0), EINVAL), (dict(G=3), EUNSUPPORTED), (dict(G=16), EUNSUPPORTED), (dict(B=65536), EUNSUPPORTED),
    (dict(C=(1 << 20) + 8), EUNSUPPORTED), (dict(N=1 << 31), EUNSUPPORTED), (dict(B=2, N=1 << 30), EUNSUPPORTED),
    (dict(row=-8), EINVAL), (dict(batch=-8), EINVAL), (dict(add=P, add_s=-1), EINVAL), (dict(scale=P, scale_s=-1), EINVAL),
    (dict(shift=P, shift_s=-1), EINVAL), (dict(x=P + 2), EALIGN), (dict(x=P + 1, dtype=1), EALIGN), (dict(out=P + 2), EALIGN),
    (dict(weight=P + 2), EALIGN), (dict(bias=P + 1), EALIGN), (dict(add=P + 2), EALIGN), (dict(offsets=P + 2), EALIGN),
    (dict(row=16), EINVAL), (dict(out=P + 32), EINVAL), (dict(out=P - 32), EINVAL), (dict(dtype=1, out_dtype=0, G=1), EINVAL),
    (dict(B=2, batch=0), EINVAL), (dict(row=0), EINVAL), (dict(row=1 << 62, out=P + 512), EINVAL),
    (dict(N=100000), EWORKSPACE), (dict(N=100000, ws=P, ws_bytes=16), EWORKSPACE), (dict(N=100000, ws=P + 8, ws_bytes=1 << 30), EWORKSPACE)])
def test_groupnorm(lib, kw, code):
    assert _norm(lib, **kw) == code
    assert b"dgq_groupnorm" in lib.dgq_last_error()


BIG = (C.c_float * 4096)()
Q = (C.addressof(BIG) + 8192 + 15) & ~15


@pytest.mark.parametrize("name,at", [(n, a) for n in ("weight", "bias", "add", "scale", "shift", "offsets") for a in (0, 252, -4)])
def test_groupnorm_into_what_it_reads(lib, name, at):
    """out has 8 rows of 8 fp32 channels: tables that begin inside it and (vectors, offsets) ones that end there."""
    size = {"weight": 32, "bias": 32, "add": 32, "scale": 32, "shift": 32, "offsets": 8}[name]
    kw = {name: Q + (at if at >= 0 else 4 - size)}
    assert _norm(lib, x=Q - 4096, out=Q, **kw) == EINVAL
    assert b"dgq_groupnorm: out overlaps " + name.encode() in lib.dgq_last_error()


def test_groupnorm_into_rows_of_a_table(lib):
    """Two images' rows of a table, 1024 floats apart, out in the second of them and between them."""
    for at in (4096, 2048):
        assert _norm(lib, x=Q - 4096, out=Q, B=2, batch=64, scale=Q - at, scale_s=1024) == EINVAL
        assert b"dgq_groupnorm: out overlaps scale" in lib.dgq_last_error()


def test_groupnorm_of_no_rows_is_no_work(lib):
    assert _norm(lib, N=0, x=None, out=None) == 0


def test_groupnorm_workspace(lib):
    size = lib.dgq_groupnorm_workspace_bytes
    assert size(2, 100000, 0, 64, 8, 0) >= 2 * 3 * 64 * 4
    for bad in ((0, 8, 0, 64, 8, 0), (1, 0, 0, 64, 8, 0), (1, 8, 0, 64, 7, 0), (1, 8, 0, 64, 8, 3)):
        assert size(*bad) == 0


@pytest.mark.parametrize("B,N,C,G,dtype", [(16384, 1, 32768, 1024, 0), (65535, 1, 32768, 512, 0), (16384, 1, 65536, 1024, 2),
                                           (4097, 129, 32768, 1024, 0), (4096, 129, 65536, 1024, 1)])
def test_groupnorm_of_more_groups_than_a_launch_takes(lib, B, N, C, G, dtype):
    """A workgroup to every group, of 256 threads or (129 rows) of 1024, would be 2^32 threads and more: such calls go through
    sums of chunks, which need a workspace.  Just below that a workgroup takes each."""
    size = lib.dgq_groupnorm_workspace_bytes
    assert size(B, N, 0, C, G, dtype) > 0
    below = B // 2 if N == 1 else 2000
    assert size(below, N, 0, C, G, dtype) == 0


@pytest.mark.parametrize("B,N,C,G,dtype,most", [(1, 1, 1 << 20, 1 << 20, 0, 16 + 12), (1, 4096, 65536, 8192, 0, 34), (1, 4096, 65536, 8192, 1, 34),
                                                (2, 500, 40000, 40, 0, 2), (1, 256, 1 << 20, 1, 0, 24), (16384, 1, 32768, 1024, 0, 257)])
def test_groupnorm_workspace_of_wide_maps(lib, B, N, C, G, dtype, most):
    """A group's channels lie in one slice of a workgroup's, or in a few neighbours: 16 bytes for each of these and each chunk of
    rows, and 12 a channel of an image where the sums are many.  most: MiB."""
    assert 0 < lib.dgq_groupnorm_workspace_bytes(B, N, 0, C, G, dtype) <= most << 20


def test_w4_bytes(lib):
    size = lib.dgq_w4_bytes
    assert size(16, 128, 128) == 1024 + 64 and size(16, 128, 32) == 1024 + 256
    assert size(17, 129, 64) == 4 * (1024 + 128) and size(1, 1, 64) == 1024 + 128
    for bad in ((0, 8, 32), (8, 0, 32), (8, 8, 16), (8, 8, 0), (8, 8, 256), ((1 << 24) + 1, 8, 32), (8, (1 << 20) + 1, 32)):
        assert size(*bad) == 0
    assert size(1 << 24, 1 << 20, 128) == (1 << 20) * (1 << 13) * 1088  # past 32 bits


@pytest.mark.parametrize("kw,code", [
    (dict(data=None), EINVAL), (dict(w=None), EINVAL), (dict(dtype=-1), EINVAL), (dict(O=0), EINVAL), (dict(C=0), EINVAL),
    (dict(row=-1), EINVAL), (dict(group=16), EUNSUPPORTED), (dict(C=(1 << 20) + 1), EUNSUPPORTED), (dict(O=(1 << 24) + 1), EUNSUPPORTED),
    (dict(O=1 << 24, C=1 << 20), EUNSUPPORTED), (dict(data=P + 8), EALIGN), (dict(w=P + 2), EALIGN), (dict(w=P + 1, dtype=2), EALIGN)])
def test_w4_pack_and_unpack(lib, kw, code):
    a = dict(w=P, dtype=0, row=8, O=8, C=8, group=32, data=P)
    a.update(kw)
    assert lib.dgq_w4_pack(a["w"], a["dtype"], a["row"], a["O"], a["C"], a["group"], a["data"], None) == code
    assert b"dgq_w4_pack" in lib.dgq_last_error()
    if "row" not in kw:
        assert lib.dgq_w4_unpack(a["data"], a["O"], a["C"], a["group"], a["dtype"], a["w"], None) == code
        assert b"dgq_w4_unpack" in lib.dgq_last_error()


@pytest.mark.parametrize("at", [0, 64, 1276, -252])
def test_w4_pack_and_unpack_into_what_they_read(lib, at):
    """8 x 8 fp32 values are 256 bytes, packed 1280: values that begin inside the packed ones, end there, or whose rows lie around
    them."""
    assert lib.dgq_w4_bytes(8, 8, 32) == 1280
    big = (C.c_float * 2048)()
    data = (C.addressof(big) + 1024 + 15) & ~15
    assert lib.dgq_w4_pack(data + at, 0, 8, 8, 8, 32, data, None) == EINVAL
    assert b"dgq_w4_pack: w overlaps data" in lib.dgq_last_error()
    assert lib.dgq_w4_unpack(data, 8, 8, 32, 0, data + at, None) == EINVAL
    assert b"dgq_w4_unpack: w overlaps data" in lib.dgq_last_error()
    assert lib.dgq_w4_pack(data - 32 - abs(at), 0, 1 << 20, 8, 8, 32, data, None) == EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(data=None), EINVAL), (dict(dtype=4), EINVAL), (dict(out_dtype=1), EINVAL),
    (dict(dtype=1, out_dtype=2), EINVAL), (dict(M=-1), EINVAL), (dict(row=-1), EINVAL), (dict(act=2), EINVAL), (dict(group=1), EUNSUPPORTED),
    (dict(M=(1 << 19) + 1), EUNSUPPORTED), (dict(x=P + 2), EALIGN), (dict(y=P + 2), EALIGN), (dict(bias=P + 2), EALIGN), (dict(data=P + 4), EALIGN),
    (dict(), EINVAL), (dict(y=P + 28), EINVAL), (dict(y=P - 28), EINVAL), (dict(M=3, row=1 << 61, y=P + 512), EINVAL),
    (dict(C=20000), EWORKSPACE), (dict(C=20000, ws=P, ws_bytes=8), EWORKSPACE), (dict(C=20000, ws=P + 4, ws_bytes=1 << 30), EWORKSPACE)])
def test_w4_matvec(lib, kw, code):
    a = dict(x=P, dtype=0, row=8, M=1, data=P, O=8, C=8, group=32, bias=None, act=0, y=P, out_dtype=0, ws=None,
             ws_bytes=0, stream=None)
    a.update(kw)
    assert lib.dgq_w4_matvec(*a.values()) == code
    assert b"dgq_w4_matvec" in lib.dgq_last_error()


@pytest.mark.parametrize("name,at", [("data", 0), ("data", 28), ("data", -1264), ("bias", 0), ("bias", 28), ("bias", -28)])
def test_w4_matvec_into_what_it_reads(lib, name, at):
    """y has 8 fp32 values; 8 x 8 weights take 1280 bytes."""
    kw = dict(data=Q - 2048, bias=None)
    y = Q + at if name == "data" and at >= 0 else Q
    kw[name] = Q if name == "data" and at >= 0 else Q - 1264 if name == "data" else Q + at
    assert lib.dgq_w4_matvec(Q + 4096, 0, 8, 1, kw["data"], 8, 8, 32, kw["bias"], 0, y, 0, None, 0, None) == EINVAL
    assert b"dgq_w4_matvec: y overlaps " + name.encode() in lib.dgq_last_error()


def test_w4_matvec_workspace(lib):
    size = lib.dgq_w4_matvec_workspace_bytes
    assert size(3, 40, 20000) % (3 * 40 * 4) == 0 and size(3, 40, 20000) > 0  # some parts of [3, 40] fp32
    assert size(3, 40, 128) == 0 and size(1, 16384, 4096) == 0
    for bad in ((0, 40, 20000), (3, 0, 20000), (3, 40, 0), (3, 40, (1 << 20) + 1)):
        assert size(*bad) == 0


def test_w4_matvec_of_no_rows_is_no_work(lib):
    assert lib.dgq_w4_matvec(None, 0, 8, 0, P, 8, 8, 32, None, 0, None, 0, None, 0, None) == 0


# ---- the references themselves ----

@pytest.mark.parametrize("group", [32, 64, 128])
def test_codes_stand_for_their_weights(group):
    """A value is off by half a scale at most (and by the cleared bits: 15 * 15 * 2^-19 scales), zero is exact."""
    rng = np.random.default_rng(1)
    w = (rng.standard_normal((33, 300)) * 2.0 ** rng.integers(-40, 40, (33, 1))).astype(np.float32)
    w[rng.random(w.shape) < 0.1] = 0
    codes, words = w4_reference.quantize(w, group)
    v = w4_reference.values(codes, words, group, 33, 300)
    s = np.repeat((words & np.uint32(0xFFFFFFF0)).view(np.float32).astype(np.float64), group, axis=1)[:33, :300]
    # a code next to 15 or 0 may be pushed past the end by the zero's own rounding: a half more
    assert (np.abs(v - w) <= s * (1 + 15 * 2.0 ** -19 + 2.0 ** -19)).all()
    assert (v[w == 0] == 0).all()


def test_groupnorm_reference():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((50, 12)).astype(np.float32)
    y, tol = norm_reference.groupnorm(x, [0, 20], [20, 45], 3, eps=0.0)
    assert np.isnan(y[45:]).all() and (tol[:45] < 1e-5).all()
    g = y[:20].reshape(20, 3, 4)
    assert np.allclose(g.mean((0, 2)), 0) and np.allclose(g.var((0, 2)), 1)
