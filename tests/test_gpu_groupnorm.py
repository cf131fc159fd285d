"""dgq_groupnorm against its definition in 64 bits (norm_reference)."""
import numpy as np
import pytest

import norm_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["fp32", "fp16", "bf16"]


@pytest.fixture(scope="module")
def dgq():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_04304_amd as m
    m.lib()
    return m


def _type(name):
    import torch
    return {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}[name]


def _map(rng, rows, C, dtype, far=1.0):
    """A convolution's output: channels of different mean and size.  The device tensor and its values."""
    import torch
    x = rng.standard_normal((rows, C)) * (0.3 + 2 * rng.random(C)) + far * rng.standard_normal(C)
    t = torch.from_numpy(x.astype(np.float32)).to(_type(dtype))
    return t.cuda(), t.float().numpy()


def _up(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _tables(rng, B, C, names):
    f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    t = dict(weight=1 + 0.2 * f(C), bias=0.2 * f(C), add=f(B, C), scale=0.5 * f(B, C), shift=0.5 * f(B, C))
    return {k: t[k] for k in names}


def _check(got, want, tol, what=""):
    got = got.float().cpu().numpy().astype(np.float64).reshape(want.shape)
    there = ~np.isnan(want)
    bad = ~(np.abs(got - want) <= tol) & there
    assert not bad.any(), "%s: %d of %d values off, first %s: %r for %r (allowed %g)" % (
        what, bad.sum(), there.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0], tol[bad][0])


def _even(B, N):
    return [i * N for i in range(B)], [(i + 1) * N for i in range(B)]


ALL = ("weight", "bias", "add", "scale", "shift")
# B, N, C, G: single values, widths that fill no vector, groups that end inside one, one image of many rows, many of few, more
# channels than one workgroup takes, maps that a workgroup holds in registers and larger ones, groups too many to be added up by all
SIZES = [(1, 1, 1, 1), (1, 1, 32, 32), (3, 1, 40, 8), (2, 7, 30, 30), (2, 64, 37, 1), (1, 100, 90, 30), (5, 33, 129, 3),
         (2, 256, 320, 32), (2, 64, 1280, 32), (1, 4099, 128, 32), (300, 3, 24, 4), (2, 50, 2560, 32), (1, 9, 5000, 8),
         (1, 5, 9001, 1), (4, 1024, 320, 32), (1, 20000, 16, 4),
         (1, 3000, 256, 256), (2, 6, 4096, 4096), (7, 600, 320, 32), (6, 2100, 320, 32), (3, 300, 516, 4), (9, 513, 264, 24),
         (2, 700, 999, 3), (1, 900, 4099, 1), (40, 300, 259, 7), (12, 64, 1926, 1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,C,G", SIZES)
def test_sizes(dgq, B, N, C, G, dtype):
    rng = np.random.default_rng(B + 10 * N + 100 * C)
    x, xn = _map(rng, B * N, C, dtype)
    t = _tables(rng, B, C, ALL)
    out = dgq.dgq_groupnorm(x.view(B, N, C), G, act=dgq.ACT_SILU, **{k: _up(v) for k, v in t.items()})
    assert out.shape == (B, N, C) and out.dtype == x.dtype
    _check(out, *ref.groupnorm(xn, *_even(B, N), G, silu=True, out_type=dtype, **t))
    out = dgq.dgq_groupnorm(x.view(B, N, C), G, dtype=_type("fp32"))
    assert out.dtype == _type("fp32")
    _check(out, *ref.groupnorm(xn, *_even(B, N), G))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,C,G", [(1, 700, 7000, 28), (2, 300, 9000, 3), (2, 40, 10007, 10007), (1, 700, 6000, 24), (3, 90, 8200, 4100),
                                     (1, 700, 20002, 73), (1, 700, 8192, 1)])
def test_groups_in_several_slices_of_the_channels(dgq, B, N, C, G, dtype):
    """More channels than a workgroup takes: groups that lie in one slice of them, that some slices cut, that cover slices; out
    of a workspace that held NaN, so that every sum that is read was written."""
    import torch
    assert C % G == 0
    rng = np.random.default_rng(C + G)
    x, xn = _map(rng, B * N, C, dtype)
    t = _tables(rng, B, C, ("weight", "add", "shift"))
    need = dgq.dgq_groupnorm_workspace_bytes(B, N, False, C, G, x.dtype)
    assert need > 0
    ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")
    for to in {dtype, "fp32"}:
        out = dgq.dgq_groupnorm(x.view(B, N, C), G, dtype=_type(to), workspace=ws, **{k: _up(v) for k, v in t.items()})
        _check(out, *ref.groupnorm(xn, *_even(B, N), G, out_type=to, **t))
    assert (ws[-16:] == 255).all()


# many rows that workgroups of 1024 threads just hold, in groups that end inside a vector and that do not
HELD = [(6, 4500, 320, 32), (8, 2500, 480, 30), (192, 1500, 48, 1)]
# packed: lengths and channels
HELD_PACKED = [([2000, 1800, 0, 2500, 4100, 1, 900, 2700], 960, 32), ([30, 8200, 6000, 3500, 1, 0], 640, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,C,G", HELD)
def test_many_rows_that_a_workgroup_holds(dgq, B, N, C, G, dtype):
    rng = np.random.default_rng(B + N)
    x, xn = _map(rng, B * N, C, dtype)
    t = _tables(rng, B, C, ("bias", "add", "scale"))
    for to in sorted({dtype, "fp32"}):
        out = dgq.dgq_groupnorm(x.view(B, N, C), G, dtype=_type(to), act=dgq.ACT_SILU, **{k: _up(v) for k, v in t.items()})
        _check(out, *ref.groupnorm(xn, *_even(B, N), G, silu=True, out_type=to, **t))
    kept = dgq.dgq_groupnorm(x.view(B, N, C), G)
    assert dgq.dgq_groupnorm(x.view(B, N, C), G, out=x.view(B, N, C)).equal(kept)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,C,G", HELD_PACKED)
def test_packed_rows_of_which_a_workgroup_holds_most(dgq, lengths, C, G, dtype):
    """Images of as many rows as a workgroup holds, fewer and more; in place and not, of x's type and fp32."""
    import torch
    rng = np.random.default_rng(sum(lengths))
    B, front, behind = len(lengths), 2, 3
    offsets = front + np.concatenate([[0], np.cumsum(lengths)])
    rows = int(offsets[-1]) + behind
    x, xn = _map(rng, rows, C, dtype)
    t = _tables(rng, B, C, ("weight", "add", "shift"))
    kw = dict(offsets=_up(offsets.astype(np.int32)), **{k: _up(v) for k, v in t.items()})
    want = {to: ref.groupnorm(xn, offsets[:-1], offsets[1:], G, out_type=to, **t) for to in {dtype, "fp32"}}
    for to in want:
        out = torch.full((rows, C), 7.0, dtype=_type(to), device="cuda")
        _check(dgq.dgq_groupnorm(x, G, out=out, **kw), *want[to])
        assert (out[:front] == 7).all() and (out[rows - behind:] == 7).all()
    kept = x.clone()
    _check(dgq.dgq_groupnorm(x, G, out=x, **kw), *want[dtype])
    assert torch.equal(x[:front], kept[:front]) and torch.equal(x[rows - behind:], kept[rows - behind:])


def test_more_groups_than_a_launch_takes(dgq):
    """2^24 groups of 32 values, through sums of chunks: 16384 images of one row and 32768 channels."""
    import torch
    B, C, G = 16384, 32768, 1024
    x = torch.empty((B, 1, C), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    x.normal_(generator=g)
    out = dgq.dgq_groupnorm(x, G)
    for b in (0, 1, 4095, 8192, B - 2, B - 1):
        xn = x[b].cpu().numpy()
        _check(out[b], *ref.groupnorm(xn, [0], [1], G), "image %d" % b)
    m = out.view(B, G, 32).double().mean(2)
    assert m.abs().max() < 1e-5  # every group of every image; 32 values of 2^-24 of 5 each


@pytest.mark.parametrize("names", [(), ("weight",), ("bias",), ("add",), ("scale",), ("shift",), ("add", "scale"),
                                   ("weight", "bias", "shift")])
@pytest.mark.parametrize("B,N,C,G", [(2, 40, 320, 32), (2, 3000, 80, 8)])
def test_what_is_not_given(dgq, names, B, N, C, G):
    rng = np.random.default_rng(5)
    x, xn = _map(rng, B * N, C, "bf16")
    t = _tables(rng, B, C, names)
    for silu in (False, True):
        out = dgq.dgq_groupnorm(x.view(B, N, C), G, act=int(silu), eps=0.1, **{k: _up(v) for k, v in t.items()})
        _check(out, *ref.groupnorm(xn, *_even(B, N), G, eps=0.1, silu=silu, out_type="bf16", **t))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths", [[0], [5], [0, 0, 0], [1, 0, 1], [700, 0, 1, 64, 3000, 2], [3, 5000], [0, 17, 0],
                                     list(range(40)), [1] * 200])
@pytest.mark.parametrize("C,G", [(96, 32), (50, 2)])
def test_packed(dgq, lengths, C, G, dtype):
    """Ragged images, empty ones; rows in front of the first and behind the last keep what out held."""
    import torch
    rng = np.random.default_rng(len(lengths) + sum(lengths))
    B, front, behind = len(lengths), 3, 2
    offsets = front + np.concatenate([[0], np.cumsum(lengths)])
    rows = int(offsets[-1]) + behind
    x, xn = _map(rng, rows, C, dtype)
    t = _tables(rng, B, C, ALL)
    out = torch.full((rows, C), 7.0, dtype=_type("fp32"), device="cuda")
    got = dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU, offsets=_up(offsets.astype(np.int32)), out=out, **{k: _up(v) for k, v in t.items()})
    assert got is out
    want, tol = ref.groupnorm(xn, offsets[:-1], offsets[1:], G, silu=True, **t)
    _check(out, want, tol)
    assert (out[:front] == 7).all() and (out[rows - behind:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("C,G", [(80, 8), (96, 8)])
def test_packed_with_one_long_image(dgq, C, G, in_place, dtype):
    """An image far longer than the others, whose rows no workgroup holds, and groups that fill no vector."""
    import torch
    rng = np.random.default_rng(C)
    lengths = [int(n) for n in rng.integers(0, 30, 40)]
    lengths[17] = 9001
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    x, xn = _map(rng, int(offsets[-1]), C, dtype)
    t = _tables(rng, 40, C, ("weight", "add", "shift"))
    out = dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU, offsets=_up(offsets.astype(np.int32)), out=x if in_place else torch.empty_like(x),
                            **{k: _up(v) for k, v in t.items()})
    _check(out, *ref.groupnorm(xn, offsets[:-1], offsets[1:], G, silu=True, out_type=dtype, **t))


@pytest.mark.parametrize("B", [63, 64, 65, 130, 4097, 9000])
def test_packed_of_many_images(dgq, B):
    """Images of 0 to 3 rows, of which a chunk holds many: the search among them takes one to three steps."""
    import torch
    rng = np.random.default_rng(B)
    C, G = 40, 20  # groups below a vector
    offsets = 3 + np.concatenate([[0], np.cumsum(rng.integers(0, 4, B))])
    rows = int(offsets[-1]) + 2
    x, xn = _map(rng, rows, C, "fp32")
    t = _tables(rng, B, C, ("weight", "add"))
    out = torch.full((rows, C), 7.0, device="cuda")
    assert dgq.dgq_groupnorm(x, G, offsets=_up(offsets.astype(np.int32)), out=out, **{k: _up(v) for k, v in t.items()}) is out
    _check(out, *ref.groupnorm(xn, offsets[:-1], offsets[1:], G, **t))
    assert (out[:3] == 7).all() and (out[-2:] == 7).all()


def test_packed_offsets_out_of_order_stay_inside(dgq):
    """Offsets below 0, above the rows and descending: wrong rows, but none outside the tensors."""
    import torch
    rng = np.random.default_rng(8)
    rows = 500
    for G, offsets in ((g, o) for g in (8, 64) for o in ([-5, 900, 20, 400, 10 ** 9], [400, 300, 200, 100, 0], [0, 500, 0, 500, 0],
                                                         [-9, -8, -7, -6, -5])):
        C = 64
        around = torch.full((rows + 200, C), 3.0, device="cuda")
        out = around[100:100 + rows]
        dgq.dgq_groupnorm(_map(rng, rows, C, "fp32")[0], G, offsets=_up(np.array(offsets, np.int32)), out=out)
        torch.cuda.synchronize()
        assert (around[:100] == 3).all() and (around[100 + rows:] == 3).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [60, 5000])
def test_strides(dgq, N, dtype):
    """x a part of wider rows at odd places, images apart; the terms columns of one projection's output."""
    import torch
    rng = np.random.default_rng(9)
    B, C, G = 2, 60, 4
    wide, _ = _map(rng, B * (N + 5), C + 11, dtype)
    x = wide.view(B, N + 5, C + 11)[:, 2:2 + N, 3:3 + C]
    xn = x.float().cpu().numpy().reshape(B * N, C)
    emb = rng.standard_normal((B, 3 * C + 1)).astype(np.float32)
    e = _up(emb)
    out = dgq.dgq_groupnorm(x, G, add=e[:, :C], scale=e[:, C:2 * C], shift=e[:, 2 * C + 1:])
    assert out.is_contiguous()
    _check(out, *ref.groupnorm(xn, *_even(B, N), G, add=emb[:, :C], scale=emb[:, C:2 * C], shift=emb[:, 2 * C + 1:], out_type=dtype))
    # one image's rows and one row of terms for all
    one = torch.as_strided(wide, (3, N, C), (0, C + 11, 1))
    row = torch.as_strided(e, (3, C), (0, 1))
    out = dgq.dgq_groupnorm(one, G, add=row)
    on = one[0].float().cpu().numpy()
    _check(out, *ref.groupnorm(np.concatenate([on] * 3), *_even(3, N), G, add=np.stack([emb[0, :C]] * 3), out_type=dtype))


@pytest.mark.parametrize("N,C", [(64, 320), (6000, 320), (50, 333), (3000, 333)])
def test_in_place_and_workspace(dgq, N, C):
    import torch
    rng = np.random.default_rng(10)
    B, G = 2, C // 10 if C == 320 else 9
    x, xn = _map(rng, B * N, C, "fp16")
    x = x.view(B, N, C)
    other = dgq.dgq_groupnorm(x, G)
    ws = torch.full((dgq.dgq_groupnorm_workspace_bytes(B, N, False, C, G, x.dtype) + 16,), 255, dtype=torch.uint8, device="cuda")
    assert dgq.dgq_groupnorm(x, G, out=x, workspace=ws) is x
    assert torch.equal(x, other)
    assert (ws[-16:] == 255).all()
    with pytest.raises(dgq.DgqError, match="workspace"):
        dgq.dgq_groupnorm(torch.zeros((2, 9000, C), device="cuda"), G, workspace=ws[:16])


@pytest.mark.parametrize("N", [64, 5000])
def test_means_far_from_zero(dgq, N):
    """Means of 10^3 deviations, and an embedding that takes them away or brings them."""
    rng = np.random.default_rng(11)
    C, G = 64, 4
    x, xn = _map(rng, N, C, "fp32", far=0.0)
    far = np.full((1, C), 1000.0, np.float32)
    y = _up((xn + far).astype(np.float32))
    yn = (xn + far).astype(np.float32)
    _check(dgq.dgq_groupnorm(y.view(1, N, C), G), *ref.groupnorm(yn, *_even(1, N), G), "far")
    _check(dgq.dgq_groupnorm(y.view(1, N, C), G, add=_up(-far)), *ref.groupnorm(yn, *_even(1, N), G, add=-far), "back")
    _check(dgq.dgq_groupnorm(x.view(1, N, C), G, add=_up(far)), *ref.groupnorm(xn, *_even(1, N), G, add=far), "there")


@pytest.mark.parametrize("N", [33, 4000])
def test_equal_values_give_the_bias(dgq, N):
    import torch
    x = torch.full((1, N, 16), 3.1, device="cuda")
    bias = _up(np.arange(16, dtype=np.float32))
    out = dgq.dgq_groupnorm(x, 2, bias=bias)
    assert torch.allclose(out, bias.expand(1, N, 16), atol=1e-4)  # 3.1 to the sums' last bits, times 1 / sqrt(eps)


@pytest.mark.parametrize("N", [33, 4000])
def test_what_is_not_finite_stays_in_its_group(dgq, N):
    rng = np.random.default_rng(12)
    B, C, G = 3, 64, 4
    x, xn = _map(rng, B * N, C, "fp32")
    want = dgq.dgq_groupnorm(x.view(B, N, C), G).cpu().numpy()
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = x.clone().view(B, N, C)
        y[1, N // 2, 17] = bad
        got = dgq.dgq_groupnorm(y, G).cpu().numpy()
        assert np.isnan(got[1, :, 16:32]).all()
        got[1, :, 16:32] = want[1, :, 16:32]
        assert np.array_equal(got, want)


def test_large_values(dgq):
    """Squares past fp32's largest number."""
    rng = np.random.default_rng(13)
    N, C, G = 200, 32, 4
    x, xn = _map(rng, N, C, "fp32")
    big = (xn * np.float32(2.0 ** 100)).astype(np.float32)
    _check(dgq.dgq_groupnorm(_up(big).view(1, N, C), G), *ref.groupnorm(big, *_even(1, N), G))


def test_far_exponents_of_silu(dgq):
    """Large values of either sign behind the norm: SiLU is 0 or the value, never NaN."""
    rng = np.random.default_rng(14)
    N, C, G = 40, 32, 4
    x, xn = _map(rng, N, C, "fp32")
    t = dict(shift=np.linspace(-500, 500, C).astype(np.float32)[None])
    _check(dgq.dgq_groupnorm(x.view(1, N, C), G, act=dgq.ACT_SILU, shift=_up(t["shift"])),
           *ref.groupnorm(xn, *_even(1, N), G, silu=True, **t))


def test_offsets_past_31_bits(dgq):
    """A strided map whose last rows lie past 2^31 elements."""
    import torch
    N, C, G, stride = 70, 64, 8, 1 << 25
    base = torch.zeros((N - 1) * stride + C, dtype=torch.float16, device="cuda")
    x = torch.as_strided(base, (1, N, C), (0, stride, 1))
    rng = np.random.default_rng(15)
    v, vn = _map(rng, N, C, "fp16")
    x.copy_(v.view(1, N, C))
    _check(dgq.dgq_groupnorm(x, G), *ref.groupnorm(vn, *_even(1, N), G, out_type="fp16"))


@pytest.mark.parametrize("N", [64, 4096])
def test_same_bits_on_streams_and_in_graphs(dgq, N):
    """Two captured calls that share one workspace, replayed with other inputs and eager calls between."""
    import torch
    rng = np.random.default_rng(16)
    B, C, G = 2, 320, 32
    x, _ = _map(rng, B * N, C, "fp32")
    x = x.view(B, N, C)
    y, _ = _map(rng, B * N, C, "fp32")
    y = y.view(B, N, C)
    ws = torch.empty(dgq.dgq_groupnorm_workspace_bytes(B, N, False, C, G, x.dtype), dtype=torch.uint8, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    want = dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU)
    with torch.cuda.stream(side):
        assert torch.equal(dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU), want)
    got = dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    graphs = []
    with torch.cuda.stream(side):
        for out in (a, b):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU, out=out, workspace=ws)
                dgq.dgq_groupnorm(out, G, out=out, workspace=ws)
            graphs.append(graph)
    torch.cuda.synchronize()
    keep = x.clone()
    for rep in range(4):
        x.copy_(y if rep % 2 else keep)
        want = dgq.dgq_groupnorm(dgq.dgq_groupnorm(x, G, act=dgq.ACT_SILU), G)
        for graph, out in zip(graphs, (a, b)):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), rep


def test_empty(dgq):
    import torch
    assert dgq.dgq_groupnorm(torch.empty((2, 0, 64), device="cuda"), 8).shape == (2, 0, 64)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert dgq.dgq_groupnorm(torch.empty((0, 64), device="cuda"), 8, offsets=off).shape == (0, 64)


@pytest.mark.parametrize("N", [0, 1, 5000])
def test_no_images(dgq, N):
    """No images are no work, as images of no rows are; what is wrong with the call is still refused."""
    import torch
    x, row = torch.empty((0, N, 64), dtype=torch.float16, device="cuda"), torch.empty((0, 64), device="cuda")
    out = dgq.dgq_groupnorm(x, 8, torch.ones(64, device="cuda"), add=row, scale=row, dtype=torch.float32)
    assert out.shape == (0, N, 64) and out.dtype == torch.float32
    assert dgq.dgq_groupnorm(x, 8, out=x) is x
    with pytest.raises(dgq.DgqError, match="multiple of G"):
        dgq.dgq_groupnorm(x, 7)
    with pytest.raises(ValueError, match="add"):
        dgq.dgq_groupnorm(x, 8, add=torch.zeros((1, 64), device="cuda"))


def test_refusals(dgq):
    import torch
    f = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    x = f(2, 10, 64)
    for kw, error, text in [
            (dict(num_groups=7), dgq.DgqError, "multiple of G"), (dict(num_groups=0), dgq.DgqError, "empty"),
            (dict(eps=-1.0), dgq.DgqError, "eps"), (dict(eps=float("nan")), dgq.DgqError, "eps"), (dict(act=2), dgq.DgqError, "act"),
            (dict(dtype=torch.float16), dgq.DgqError, "out_dtype"), (dict(dtype=torch.int32), ValueError, "dtype"),
            (dict(dtype=3), TypeError, "dtype"), (dict(weight=f(63)), ValueError, "weight"),
            (dict(weight=f(64, dtype=torch.float16)), TypeError, "weight"), (dict(bias=f(65)), ValueError, "bias"),
            (dict(add=f(3, 64)), ValueError, "add"), (dict(scale=f(2, 63)), ValueError, "scale"), (dict(shift=f(64)), ValueError, "shift"),
            (dict(add=f(2, 128)[:, ::2]), TypeError, "add"), (dict(add=f(2, 64, dtype=torch.float16)), TypeError, "add"),
            (dict(out=f(2, 10, 63)), ValueError, "out"), (dict(out=f(2, 64, 10).transpose(1, 2)), TypeError, "out"),
            (dict(out=f(2, 20, 64)[:, :10]), ValueError, "out"), (dict(x=f(20, 64)), ValueError, "x must have 3"),
            (dict(x=f(2, 64, 10).transpose(1, 2)), TypeError, "x must be"), (dict(x=x.cpu()), TypeError, "x must be"),
            (dict(x=x.double()), TypeError, "x must be"), (dict(offsets=f(3, dtype=torch.int32)), ValueError, "x must have 2"),
            (dict(x=f(20, 64), offsets=f(3)), TypeError, "offsets"), (dict(x=f(20, 64), offsets=f(1, dtype=torch.int32)), dgq.DgqError, "empty"),
            (dict(x=f(20, 64), offsets=f(0, dtype=torch.int32)), ValueError, "offsets"), (dict(weight=torch.zeros(64)), TypeError, "weight")]:
        args = dict(x=x, num_groups=8)
        args.update(kw)
        with pytest.raises(error, match=text):
            dgq.dgq_groupnorm(**args)
