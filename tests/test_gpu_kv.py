"""The 8-bit cache of text keys and values and the attention that reads it, against their plain forms in kv_reference."""
import numpy as np
import pytest

import kv_reference as ref

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


def _i32(v):
    import torch
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _floats(rng, shape, dtype, spread=True):
    """A device tensor of `dtype` and its values in fp32 numpy."""
    import torch
    x = rng.standard_normal(shape).astype(np.float32)
    if spread:
        x *= (0.25 + rng.random(shape[-2:])).astype(np.float32)
    t = torch.from_numpy(x).to(_type(dtype))
    return t.cuda(), t.float().numpy()


# ---- planning --------------------------------------------------------------------------------------------------------

def _check_plan(dgq, lengths, new, table, free, n_free, S, rows):
    import torch
    want = ref.plan(lengths, new, table, free, n_free, S, rows)
    t = _i32(table)
    state = [_i32(lengths), _i32(new), _i32(free), _i32([n_free])]
    kept = [x.clone() for x in state]
    p = dgq.dgq_kv_plan(state[0], state[1], t, state[2], state[3], S, rows)
    torch.cuda.synchronize()
    runs = p.runs.cpu().numpy()
    assert np.array_equal(t.cpu().numpy(), want[0])
    assert p.lengths.tolist() == [int(x) for x in want[1]]
    assert p.n_free.tolist() == [want[2]]
    assert p.row_offsets.tolist() == want[3]
    assert p.counts.tolist() == want[5]
    assert runs.shape == (rows // S + 2 * len(lengths), 4)
    assert [tuple(r) for r in runs[:len(want[4])]] == [tuple(int(x) for x in r) for r in want[4]]
    assert (runs[len(want[4]):] == [-1, 0, 0, 0]).all()
    assert all(torch.equal(a, b) for a, b in zip(state, kept))


@pytest.mark.parametrize("S", [32, 64, 128])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 1023, 1025, 4096])
def test_plan(dgq, B, S):
    rng = np.random.default_rng(B * 7 + S)
    W = 6
    lengths = rng.integers(0, 3 * S + 1, B)
    lengths[rng.random(B) < 0.3] = S * rng.integers(0, 3)  # blocks that are just full, and none
    new = rng.integers(0, 3 * S + 1, B)
    new[rng.random(B) < 0.3] = rng.choice([0, 1, S, S - 1])
    free = rng.permutation(B * W + 5)
    table = rng.integers(0, 99999, (B, W))
    _check_plan(dgq, lengths, new, table, free, B * W, S, int(new.sum()))
    _check_plan(dgq, lengths, new, table, free, B * W // 4, S, int(new.sum()))        # the free blocks run out
    _check_plan(dgq, lengths, new, table, free, B * W, S, int(new.sum()) * 2 // 3)    # the packed rows end early


def test_plan_of_what_cannot_be_served(dgq):
    S, W = 32, 4
    table = np.arange(28).reshape(7, W)
    free = np.arange(100, 140)
    # too long by a row; negative on either side; nothing to add; one that still fits
    lengths, new = [0, 128, -5, 10, 0, 127, 3], [129, 1, 3, -4, 0, 1, 2]
    _check_plan(dgq, lengths, new, table, free, 40, S, 500)
    _check_plan(dgq, lengths, new, table, free, 0, S, 500)
    # more free blocks than the list has room for, and fewer than none
    _check_plan(dgq, [0], [100], table[:1], free, 1000, S, 100)
    _check_plan(dgq, [0], [100], table[:1], free, -3, S, 100)
    _check_plan(dgq, [0, 5, 0], [0, 0, 0], table[:3], free, 9, S, 0)


def test_plan_counts_beyond_31_bits(dgq):
    """Rows that are asked for past 2^31 are refused; the offsets that cannot be told stay at the largest number."""
    import torch
    big = 2 ** 31 - 1
    t = _i32(np.zeros((4, 4)))
    p = dgq.dgq_kv_plan(_i32([0, big, 0, 0]), _i32([5, big, big, 7]), t, _i32(np.arange(9)), _i32([9]), 32, 1000)
    torch.cuda.synchronize()
    assert p.lengths.tolist() == [5, big, 0, 0] and p.counts.tolist()[:3] == [1, 1, 3]
    assert p.row_offsets.tolist() == [0, 5, big, big, big]
    assert p.runs[0].tolist() == [8, 0, 0, 5] and p.runs[1].tolist() == [-1, 0, 0, 0]


def test_plan_of_one_long_request(dgq):
    S, W = 32, 3000
    free = np.random.default_rng(0).permutation(4000)
    _check_plan(dgq, [45], [2900 * 32 + 1], np.zeros((1, W), int), free, 4000, S, 2900 * 32 + 1)


@pytest.mark.parametrize("B", [1, 64, 1500, 4096])
def test_release(dgq, B):
    import torch
    rng = np.random.default_rng(B)
    S, W = 64, 5
    lengths = rng.integers(-3, W * S + 100, B)
    done = (rng.random(B) < 0.5).astype(np.uint8) * 3
    table = rng.integers(0, 10 ** 6, (B, W))
    n_free = 4
    want, want_lengths = ref.release(done, lengths, table, [7, 8, 9, 10], n_free, S)
    for capacity in (B * W + 10, max(5, len(want) - 3)):  # room for all, and a list that would overflow
        free = np.full(capacity, -7)
        free[:4] = [7, 8, 9, 10]
        f = _i32(free)
        n, m = dgq.dgq_kv_release(torch.from_numpy(done).cuda(), _i32(lengths), _i32(table), f, _i32([n_free]), S)
        torch.cuda.synchronize()
        n_out = min(len(want), capacity)
        assert n.tolist() == want_lengths and m.tolist() == [n_out]
        got = f.cpu().numpy()
        assert got[:n_out].tolist() == want[:n_out] and (got[n_out:] == -7).all()


# ---- writing and reading back ------------------------------------------------------------------------------------------

def _cache(dgq, n_blocks, S, H, d, fill=0xA5):
    import torch
    c = dgq.KVCache.empty(n_blocks, S, H, d)
    c.data.fill_(fill)
    assert c.data.dtype == torch.uint8
    return c


def _read(c):
    return ref.Cache(c.data.cpu().numpy(), c.n_blocks, c.block_size, c.heads, c.d)


def _same_cache(got, want, blocks):
    for b in blocks:
        assert np.array_equal(got.scales[b].view(np.uint32), want.scales[b].view(np.uint32)), b
        for w in range(2):
            assert np.array_equal(got.codes[w][b], want.codes[w][b]), (b, w)
            assert (got.padding[w][b] == 128).all(), (b, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S,H,d", [(32, 1, 8), (32, 3, 40), (64, 2, 64), (64, 5, 72), (128, 2, 128), (128, 1, 248), (32, 2, 256)])
def test_store(dgq, dtype, S, H, d):
    import torch
    rng = np.random.default_rng(S + d)
    n_blocks, rows = 9, 3 * S + 40
    k, kn = _floats(rng, (rows, H, d), dtype)
    v, vn = _floats(rng, (rows, H, d), dtype)
    c = _cache(dgq, n_blocks, S, H, d)
    before = c.data.clone()
    # whole blocks, parts of them, one row, rows out of order; then pieces that continue blocks
    first = [(4, 0, 0, S), (0, S, 0, 7), (7, S + 7, 0, 1), (3, 3 * S, 0, 40 if S > 40 else S - 1)]
    then = [(0, 2 * S, 7, S - 7), (7, 20, 1, 5), (3, 3, S - 1, 1)]
    want = _read(c)
    for runs in (first, then):
        padded = runs + [(-1, 0, 0, 0)] * 3
        dgq.dgq_kv_store(c, k, v, _i32(padded))
        torch.cuda.synchronize()
        ref.store(want, kn, vn, runs)
        _same_cache(_read(c), want, [r[0] for r in runs])
    # the blocks that no run names keep every byte
    e, other = -(-d // 16) * 16, [1, 2, 5, 6, 8]
    n = n_blocks * H * S * 2 * e
    for x, y in ((c.data[:n], before[:n]), (c.data[n:], before[n:])):
        assert torch.equal(x.view(n_blocks, -1)[other], y.view(n_blocks, -1)[other])
    # and the same call again leaves the same bytes
    again = c.data.clone()
    dgq.dgq_kv_store(c, k, v, _i32(then))
    torch.cuda.synchronize()
    assert torch.equal(again, c.data)


@pytest.mark.parametrize("dtype", TYPES)
def test_store_of_views(dgq, dtype):
    """K and V of one stacked projection, and every second head of a wider tensor."""
    import torch
    rng = np.random.default_rng(3)
    rows, H, d, S = 50, 4, 24, 32
    x, xn = _floats(rng, (rows, 3, H, d), dtype)
    y, yn = _floats(rng, (rows, 2 * H, d), dtype)
    for k, v, kn, vn in ((x[:, 1], x[:, 2], xn[:, 1], xn[:, 2]), (x[:, 0], y[:, 1::2], xn[:, 0], yn[:, 1::2])):
        c = _cache(dgq, 3, S, H, d)
        want = _read(c)
        runs = [(2, 0, 0, 32), (0, 32, 0, 18)]
        dgq.dgq_kv_store(c, k, v, _i32(runs))
        torch.cuda.synchronize()
        ref.store(want, np.ascontiguousarray(kn), np.ascontiguousarray(vn), runs)
        _same_cache(_read(c), want, [2, 0])


def test_store_of_zeros_and_of_what_is_not_finite(dgq):
    import torch
    rng = np.random.default_rng(4)
    H, d, S = 6, 16, 32
    k, kn = _floats(rng, (20, H, d), "fp32")
    k[:, 0] = 0
    k[:, 1] *= 2.0 ** -100                      # below the least scale: zeros
    k[:, 2] *= 1e-25                            # small, but held
    k[3, 3, 5] = float("nan")
    k[3, 4, 5] = float("inf")
    k[3, 5, 5] = 3e38
    c = _cache(dgq, 2, S, H, d)
    runs = [(1, 0, 0, 20)]
    want = _read(c)
    dgq.dgq_kv_store(c, k, k, _i32(runs))
    torch.cuda.synchronize()
    got = _read(c)
    kn = k.cpu().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        ref.store(want, kn, kn, runs)
    for h in (0, 1, 2, 5):
        assert got.scales[1, h].tolist() == want.scales[1, h].tolist()
        assert np.array_equal(got.codes[0][1][:, h], want.codes[0][1][:, h])
    assert (got.scales[1, :2] == 0).all() and (got.codes[0][1][:, :2] == 0).all()
    assert np.isnan(got.scales[1, 3]).all() and np.isinf(got.scales[1, 4]).all()
    assert (got.codes[0][1][:, 3:5] == 0).all()
    # rows added to such blocks: a zero block takes their scale, one that is not finite stays so
    ok, okn = _floats(rng, (1, H, d), "fp32")
    dgq.dgq_kv_store(c, ok, ok, _i32([(1, 0, 20, 1)]))
    torch.cuda.synchronize()
    got = _read(c)
    assert (got.scales[1, 0] == np.abs(okn[0, 0]).max() * (np.float32(1) / np.float32(127))).all()
    assert np.isnan(got.scales[1, 3]).all() and np.isinf(got.scales[1, 4]).all()


def test_runs_that_point_nowhere_are_passed_over(dgq):
    import torch
    H, d, S = 2, 16, 32
    k, _ = _floats(np.random.default_rng(1), (40, H, d), "fp16")
    c = _cache(dgq, 2, S, H, d)
    before = c.data.clone()
    big = 2 ** 31 - 1
    bad = [(2, 0, 0, 4), (-1, 0, 0, 4), (big, 0, 0, 4), (0, 0, 30, 3), (0, 0, -1, 3), (0, 38, 0, 3), (0, -1, 0, 3), (0, 0, 0, 0),
           (0, 0, 0, -2), (0, big, 0, 5), (0, 0, big, 5), (0, 0, 0, big)]
    dgq.dgq_kv_store(c, k, k, _i32(bad))
    torch.cuda.synchronize()
    assert torch.equal(c.data, before)
    dgq.dgq_kv_store(c, k[:0], k[:0], _i32([(0, 0, 0, 1)]))
    dgq.dgq_kv_store(c, k, k, _i32(np.zeros((0, 4))))
    torch.cuda.synchronize()
    assert torch.equal(c.data, before)


def _filled(dgq, rng, lengths, S, H, d, dtype="fp32", W=None, spare=2, gain=None):
    """A cache with rows for every request, its table and what it holds."""
    import torch
    count = [-(-n // S) for n in lengths]
    n_blocks = sum(count) + spare
    W = W or max(1, max(count) + 1)
    ids = rng.permutation(n_blocks)
    table = np.full((len(lengths), W), -1)
    at = 0
    for b, n in enumerate(count):
        table[b, :n] = ids[at:at + n]
        at += n
    c = _cache(dgq, n_blocks, S, H, d)
    rows = sum(lengths)
    if rows:
        k, v = (_floats(rng, (rows, H, d), dtype)[0] for _ in range(2))
        if gain is not None:
            k, v = gain(k, v)
        runs, row = [], 0
        for b, n in enumerate(lengths):
            for r in range(0, n, S):
                runs.append((table[b, r // S], row + r, 0, min(S, n - r)))
            row += n
        dgq.dgq_kv_store(c, k, v, _i32(runs))
        torch.cuda.synchronize()
    return c, table, _read(c)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S,H,d", [(32, 3, 40), (64, 2, 64), (128, 1, 136), (32, 1, 256)])
def test_load(dgq, dtype, S, H, d):
    import torch
    rng = np.random.default_rng(d)
    lengths = [0, 1, S, S + 1, 2 * S - 3, 77]
    c, table, held = _filled(dgq, rng, lengths, S, H, d)
    for rows in (1, 31, 77, 3 * S):
        k, v = dgq.dgq_kv_load(c, _i32(table), _i32(lengths), rows, dtype=_type(dtype))
        torch.cuda.synchronize()
        for which, x in ((0, k), (1, v)):
            assert x.shape == (len(lengths), rows, H, d) and x.dtype == _type(dtype)
            want = np.zeros(x.shape, np.float32)
            for b, n in enumerate(lengths):
                for r in range(min(n, rows)):
                    want[b, r] = held.values(which, table[b, r // S], r % S)
            assert torch.equal(x.cpu(), torch.from_numpy(want).to(_type(dtype)))


def test_load_of_blocks_that_are_not_there(dgq):
    import torch
    rng = np.random.default_rng(5)
    c, table, held = _filled(dgq, rng, [100, 64, 10], 32, 2, 24)
    table[0, 1], table[1, 0] = c.n_blocks, -1
    k, v = dgq.dgq_kv_load(c, _i32(table), _i32([100, 1000, -4]), 160)
    torch.cuda.synchronize()
    assert (k[0, 32:64] == 0).all() and (k[1, :32] == 0).all() and (k[2] == 0).all() and (v[0, 100:] == 0).all()
    assert np.array_equal(k[0, 70].cpu().numpy(), held.values(0, table[0, 2], 6))
    assert np.array_equal(v[1, 40].cpu().numpy(), held.values(1, table[1, 1], 8))
    assert dgq.dgq_kv_load(c, _i32(table), _i32([1, 1, 1]), 0)[0].shape == (3, 0, 2, 24)


# ---- the attention -----------------------------------------------------------------------------------------------------

def _check_attention(held, table, lengths, qs, got, dtype, d):
    """got, qs: per request, fp32 numpy [n, Hq, d]"""
    for b, n in enumerate(lengths):
        k, v = ((held.exact(w, table, b, n) if n else np.zeros((0, held.codes[0].shape[2], d))) for w in (0, 1))
        want, big = ref.attention(qs[b].astype(np.float64), k, v)
        if n == 0:
            assert (got[b] == 0).all(), b
            continue
        lim = ref.tolerance(dtype, d, n, big, v, want)
        err = np.abs(got[b].astype(np.float64) - want)
        assert (err <= lim).all(), (b, n, float((err / lim).max()))


SHAPES = [  # S, H, G, d, N, lengths
    (32, 2, 1, 8, 5, [1, 0, 33]),
    (32, 8, 1, 40, 64, [77, 154]),
    (64, 3, 2, 64, 33, [1, 2, 31, 32, 33, 63, 64, 65, 231]),
    (128, 2, 1, 72, 31, [127, 128, 129, 300]),
    (32, 1, 7, 80, 20, [50, 0, 4]),
    (64, 2, 4, 128, 1, [1, 700, 0, 129]),
    (32, 1, 1, 160, 130, [77, 1]),
    (64, 1, 3, 96, 11, [400]),
    (64, 1, 1, 176, 40, [90, 17]),
    (128, 1, 2, 200, 17, [140]),
    (32, 1, 1, 256, 65, [77, 32]),
    (32, 1, 1, 224, 3, [200]),
    (32, 8, 1, 16, 1, [9000, 8193, 8192, 40] + [0, 1] * 48),  # the longest part of a split, 64 blocks to a wavefront
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "S%d_H%d_G%d_d%d_N%d" % s[:5])
def test_attention(dgq, shape, dtype):
    import torch
    S, H, G, d, N, lengths = shape
    rng = np.random.default_rng(d + N)
    c, table, held = _filled(dgq, rng, lengths, S, H, d)
    q, qn = _floats(rng, (len(lengths), N, H * G, d), dtype)
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths))
    torch.cuda.synchronize()
    assert out.shape == q.shape and out.dtype == q.dtype
    _check_attention(held, table, lengths, qn, out.float().cpu().numpy(), dtype, d)
    # the same bits again, into a buffer that held something else
    other = torch.full_like(q, float("nan"))
    assert dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), out=other) is other
    torch.cuda.synchronize()
    assert torch.equal(out, other)


MANY = [  # at least 256 workgroups of 128 rows, from one slot to several look-ups of 64 blocks; every step of the head width; both
          # kernels for many rows
    (32, 32, 1, 8, 270, [1, 0, 33]),
    (32, 8, 1, 40, 2100, [77, 154]),
    (64, 10, 1, 64, 400, [1, 2, 31, 32, 65, 231, 0]),
    (128, 4, 7, 96, 333, [127, 300, 129, 64]),
    (32, 2, 4, 128, 4200, [70]),
    (64, 8, 1, 160, 2050, [77, 95]),
    (32, 33, 1, 192, 513, [40, 5]),
    (32, 16, 2, 224, 1025, [50]),
    (64, 64, 1, 256, 257, [65, 130]),
    (32, 1, 1, 16, 33000, [4200]),
    (32, 2, 1, 32, 16500, [31]),
    (64, 8, 1, 64, 4096, [77]),
    (64, 3, 1, 96, 11100, [60]),       # one block a request, of which the table has no other
    (32, 6, 2, 120, 2800, [32, 0]),
    (32, 40, 1, 152, 901, [30]),
    (32, 32, 1, 192, 1030, [1]),
    (32, 16, 1, 216, 2060, [25]),
    (32, 9, 4, 256, 1000, [17]),
]


def width_of(S, lengths):
    """A column more than the lengths need, or the one that is enough for all."""
    return 1 if max(lengths) <= S else -(-max(lengths) // S) + 1


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "S%d_H%d_G%d_d%d_N%d" % s[:5])
def test_attention_of_many_rows(dgq, shape, dtype):
    import torch
    S, H, G, d, N, lengths = shape
    rng = np.random.default_rng(d + N)
    c, table, held = _filled(dgq, rng, lengths, S, H, d, W=width_of(S, lengths))
    q, qn = _floats(rng, (len(lengths), N, H * G, d), dtype)
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths))
    again = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), out=torch.full_like(q, float("nan")))
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    got = out.float().cpu().numpy()
    rows = np.unique(np.r_[0:40, rng.integers(0, N, 200), N - 140:N])  # whole tiles at both ends, and some between
    _check_attention(held, table, lengths, qn[:, rows], got[:, rows], dtype, d)


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_queries(dgq, dtype):
    """Requests with different numbers of queries, none among them; rows of no request keep what was there."""
    import torch
    rng = np.random.default_rng(8)
    S, H, G, d = 32, 2, 3, 48
    lengths = [40, 0, 77, 5, 100, 64]
    n = [17, 3, 0, 1, 70, 33]
    c, table, held = _filled(dgq, rng, lengths, S, H, d)
    starts = np.concatenate([[4], 4 + np.cumsum(n)])
    q, qn = _floats(rng, (starts[-1] + 5, H * G, d), dtype)
    out = torch.full_like(q, 7.0)
    dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), q_offsets=_i32(starts), out=out)
    torch.cuda.synchronize()
    assert (out[:4] == 7).all() and (out[starts[-1]:] == 7).all()
    on = out.float().cpu().numpy()
    per = lambda x: [x[starts[b]:starts[b + 1]] for b in range(len(n))]  # noqa: E731
    _check_attention(held, table, lengths, per(qn), per(on), dtype, d)
    # the same rows as a call of their own give the same numbers, to the sums' order where the split differs
    one = dgq.dgq_xattn_kv(q[None, starts[4]:starts[5]].contiguous(), c, _i32(table[4:5]), _i32(lengths[4:5]))
    torch.cuda.synchronize()
    _check_attention(held, table[4:5], lengths[4:5], [qn[starts[4]:starts[5]]], one.float().cpu().numpy(), dtype, d)


@pytest.mark.parametrize("H", [1, 4])
def test_many_packed_requests(dgq, H):
    """More requests than a wavefront looks through at once, most of them with a query or none; with four heads enough of
    them for the kernel of many rows."""
    import torch
    rng = np.random.default_rng(9)
    S, d, B = 32, 16, 200
    lengths = [int(x) for x in rng.integers(0, 40, B)]
    n = [int(x) for x in rng.choice([0, 1, 1, 2, 40], B)]
    n[60:130] = [0] * 70
    if H > 1:
        n[3], n[140], n[199] = 2000, 400, 1500
    c, table, held = _filled(dgq, rng, lengths, S, H, d)
    starts = np.concatenate([[0], np.cumsum(n)])
    q, qn = _floats(rng, (starts[-1], H, d), "fp32")
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), q_offsets=_i32(starts)).cpu().numpy()
    _check_attention(held, table, lengths, [qn[starts[b]:starts[b + 1]] for b in range(B)],
                     [out[starts[b]:starts[b + 1]] for b in range(B)], "fp32", d)


def test_offsets_that_make_no_sense_stay_in_bounds(dgq):
    import torch
    rng = np.random.default_rng(10)
    c, table, _ = _filled(dgq, rng, [40, 50, 60], 32, 1, 16)
    q, _ = _floats(rng, (20, 1, 16), "fp16")
    for starts in ([0, 2 ** 31 - 1, -5, 10], [-2 ** 31, 100, 3, 2], [20, 10, 5, 0], [7, 7, 7, 7]):
        out = torch.zeros_like(q)
        dgq.dgq_xattn_kv(q, c, _i32(table), _i32([40, 50, 60]), q_offsets=_i32(starts), out=out)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,N,H,G,d,lengths", [(1, 1, 1, 1, 64, [5000]), (2, 3, 2, 4, 128, [1, 3001]), (3, 1, 2, 1, 40, [900, 0, 128]),
                                               (1, 2, 1, 5, 256, [2047])])
def test_few_queries_over_long_rows(dgq, dtype, B, N, H, G, d, lengths):
    """Shapes whose rows are split over the chip and joined."""
    import torch
    rng = np.random.default_rng(N + d)
    c, table, held = _filled(dgq, rng, lengths, 64, H, d)
    assert dgq.dgq_xattn_kv_workspace_bytes(B, N, False, H * G, H, d, table.shape[1], 64) > 0
    q, qn = _floats(rng, (B, N, H * G, d), dtype)
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths))
    torch.cuda.synchronize()
    _check_attention(held, table, lengths, qn, out.float().cpu().numpy(), dtype, d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,lengths", [(64, [20000, 530]), (8, [140000]), (256, [6000, 5000]), (128, [7000, 100, 2100]),
                                       (256, [4000, 1]), (40, [8100, 512, 513])])
def test_packed_rows_of_many_splits(dgq, dtype, d, lengths):
    """Two to hundreds of splits, by every join; requests of one split beside them; rows of no request stay as they were."""
    import torch
    rng = np.random.default_rng(d)
    B, H, G = len(lengths), 1, 3
    c, table, held = _filled(dgq, rng, lengths, 64, H, d)
    starts = [1 + 2 * b for b in range(B + 1)]
    n = starts[-1] + 1
    q, qn = _floats(rng, (n, H * G, d), dtype)
    assert dgq.dgq_xattn_kv_workspace_bytes(B, n, True, H * G, H, d, table.shape[1], 64) > 0
    out = torch.full_like(q, 7.0)
    dgq.dgq_xattn_kv(q, c, _i32(table), _i32(lengths), q_offsets=_i32(starts), out=out)
    out = out.float().cpu().numpy()
    assert (out[0] == 7).all() and (out[-1] == 7).all()
    at = [slice(*s) for s in zip(starts, starts[1:])]
    _check_attention(held, table, lengths, [qn[s] for s in at], [out[s] for s in at], dtype, d)


@pytest.mark.parametrize("N", [1, 70, 5500])
def test_lengths_and_blocks_that_are_not_there(dgq, N):
    """Lengths past the table and below zero, blocks outside the cache: those rows are not there."""
    import torch
    rng = np.random.default_rng(12)
    S, H, d = 32, 2, 32
    c, table, held = _filled(dgq, rng, [96, 64, 64], S, H, d, W=3)
    q, qn = _floats(rng, (3, N, H, d), "fp32")
    bad = table.copy()
    bad[0, 1], bad[1, 0], bad[1, 1] = c.n_blocks, -1, 2 ** 31 - 1
    out = dgq.dgq_xattn_kv(q, c, _i32(bad), _i32([2 ** 31 - 1, 64, -1])).cpu().numpy()
    kv = [held.exact(w, table, 0, 96)[np.r_[0:32, 64:96]] for w in (0, 1)]
    want, big = ref.attention(qn[0].astype(np.float64), *kv)
    assert (np.abs(out[0] - want) <= ref.tolerance("fp32", d, 64, big, kv[1], want)).all()
    assert (out[1] == 0).all() and (out[2] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [40, 128, 160, 256])
@pytest.mark.parametrize("N,lengths", [(33, [600, 417]), (2, [1900, 1000]), (1100, [70, 90])])
def test_blocks_that_are_not_there_at_every_width(dgq, dtype, d, N, lengths):
    """Every third block is missing, in the middle of what a wavefront walks through and at its end."""
    import torch
    rng = np.random.default_rng(d + N)
    S, H = 32, 8
    c, table, held = _filled(dgq, rng, lengths, S, H, d)
    bad = table.copy()
    bad[:, 2::3] = -1
    q, qn = _floats(rng, (2, N, H, d), dtype)
    out = dgq.dgq_xattn_kv(q, c, _i32(bad), _i32(lengths)).float().cpu().numpy()
    rows = np.unique(np.r_[0:33, N - 40:N].clip(0, N - 1))
    for b, n in enumerate(lengths):
        there = np.arange(n) // S % 3 != 2
        k, v = (held.exact(w, table, b, n)[there] for w in (0, 1))
        want, big = ref.attention(qn[b][rows].astype(np.float64), k, v)
        err = np.abs(out[b][rows].astype(np.float64) - want)
        assert (err <= ref.tolerance(dtype, d, int(there.sum()), big, v, want)).all(), (b, float(err.max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,n", [(40, 300), (1, 2000), (16500, 300)])
def test_blocks_of_very_different_scales(dgq, dtype, N, n):
    """Values that grow and shrink by 2^40 from block to block, among them blocks of zeros, with all weight on any of them."""
    import torch
    rng = np.random.default_rng(n)
    S, H, d = 32, 2, 32

    def gain(k, v):
        f = torch.tensor([2.0 ** e for e in rng.integers(-40, 41, n // S + 1)], dtype=torch.float32, device="cuda")
        f[::4] = 0
        v = v * f.repeat_interleave(S)[:n, None, None]
        k = k * 3
        k[64:96] = 0
        return k, v
    c, table, held = _filled(dgq, rng, [n], S, H, d, gain=gain)
    q, qn = _floats(rng, (1, N, H, d), dtype)
    q, qn = q * 4, qn * 4
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32([n])).float().cpu().numpy()
    k, v = (held.exact(w, table, 0, n) for w in (0, 1))
    want, big = ref.attention(qn[0].astype(np.float64), k, v)
    # the bound in units of what a row adds most to this output
    for i in range(0, N, max(1, N // 60)):
        for h in range(H):
            x = k[:, h] @ qn[0, i, h] / np.sqrt(d)
            p = np.exp(x - x.max())
            most = (p / p.sum() * np.abs(v[:, h]).max(1)).max() * n
            w = np.clip(want[i, h], -65504, 65504) if dtype == "fp16" else want[i, h]
            lim = ref.tolerance(dtype, d, n, big, np.array([most]), w, shift=64)
            err = np.abs((np.clip(out[0, i, h], -65504, 65504) if dtype == "fp16" else out[0, i, h]) - w)
            assert (err <= lim).all(), (i, h, float((err / lim).max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,n", [(40, 100), (2, 900), (16500, 100)])
def test_sharp_and_extreme_queries(dgq, dtype, N, n):
    """Logits in the hundreds, queries near the types' ends, zeros; a query that is not finite spoils itself alone."""
    import torch
    rng = np.random.default_rng(13)
    S, H, d = 64, 2, 64
    c, table, held = _filled(dgq, rng, [n], S, H, d)
    q, _ = _floats(rng, (1, N, H, d), "fp32")
    q[0, 0] *= 40
    q[0, 1] = 0
    if N > 4:
        q[0, 2] *= 1e-6
        q[0, 3] *= 3e4 if dtype == "fp16" else 1e30
        q[0, 4, 0, 5] = float("nan")
        q[0, 5, 1, 63] = float("inf")
        q[0, 6, 0, 0] = float("-inf")
    q = q.clamp(-65504, 65504).to(_type(dtype)) if dtype == "fp16" else q.to(_type(dtype))
    if N > 4:
        q[0, 5, 1, 63] = float("inf")
        q[0, 6, 0, 0] = float("-inf")
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32([n])).float().cpu().numpy()
    qn = q.float().cpu().numpy()
    bad = {(4, 0), (5, 1), (6, 0)} if N > 4 else set()
    k, v = (held.exact(w, table, 0, n) for w in (0, 1))
    for i in [*range(min(N, 40)), *range(40, N, 500)]:
        for h in range(H):
            if (i, h) in bad:
                assert np.isnan(out[0, i, h]).all()
                continue
            want, big = ref.attention(qn[0, i:i + 1, h:h + 1].astype(np.float64), k[:, h:h + 1], v[:, h:h + 1])
            if big > 1e20:  # the bound says nothing there: the largest logit's row takes all
                best = np.argmax(k[:, h] @ qn[0, i, h].astype(np.float64))
                assert np.abs(out[0, i, h] - v[best, h]).max() <= 2.0 ** -7 * np.abs(v[best, h]).max()
                continue
            lim = ref.tolerance(dtype, d, n, big, v[:, h], want[0, 0])
            assert (np.abs(out[0, i, h] - want[0, 0]) <= lim).all(), (i, h)


@pytest.mark.parametrize("N", [4, 5500])
def test_rows_of_a_block_that_is_not_finite(dgq, N):
    """NaN in one request's block stays with that request and head."""
    import torch
    rng = np.random.default_rng(14)

    def gain(k, v):
        v[70, 1, 3] = float("nan")
        return k, v
    c, table, held = _filled(dgq, rng, [40, 40, 40], 32, 2, 16, gain=gain)
    q, qn = _floats(rng, (3, N, 2, 16), "fp32")
    out = dgq.dgq_xattn_kv(q, c, _i32(table), _i32([40] * 3)).cpu().numpy()
    assert np.isnan(out[1, :, 1]).all() and np.isfinite(out[[0, 2]]).all() and np.isfinite(out[1, :, 0]).all()


@pytest.mark.parametrize("N", [9, 33000])
def test_what_stands_behind_a_request_does_not_matter(dgq, N):
    """Slots behind the length hold what a former owner of the block left: large values."""
    import torch
    rng = np.random.default_rng(15)
    S, H, d = 64, 1, 32
    c, table, held = _filled(dgq, rng, [128], S, H, d, gain=lambda k, v: (k * 100, v * 100))
    q, qn = _floats(rng, (1, N, H, d), "fp32", spread=False)
    for n in (1, 31, 33, 64, 65, 100):
        out = dgq.dgq_xattn_kv(q * 0.01, c, _i32(table), _i32([n])).cpu().numpy()
        k, v = (held.exact(w, table, 0, n) for w in (0, 1))
        want, big = ref.attention((q * 0.01).cpu().numpy()[0].astype(np.float64), k, v)
        assert (np.abs(out[0] - want) <= ref.tolerance("fp32", d, n, big, v, want)).all(), n


@pytest.mark.parametrize("dtype", TYPES)
def test_strided_queries(dgq, dtype):
    """Queries that are a view of a stacked projection, [B, N, 3, H, d], and of a batch with rows between."""
    import torch
    rng = np.random.default_rng(16)
    lengths = [50, 77]
    c, table, held = _filled(dgq, rng, lengths, 32, 3, 40)
    x, xn = _floats(rng, (2, 37, 3, 3, 40), dtype)
    t, n = _i32(table), _i32(lengths)
    a = dgq.dgq_xattn_kv(x[:, :, 1], c, t, n)
    b = dgq.dgq_xattn_kv(x[:, :, 1].contiguous(), c, t, n)
    s = dgq.dgq_xattn_kv(x[:, ::2, 1], c, t, n)
    p = dgq.dgq_xattn_kv(x[:, :, 1].transpose(0, 1).reshape(74, 3, 40)[::2], c, t, n, q_offsets=_i32([0, 20, 37]))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(s, b[:, ::2])
    xs = xn[:, :, 1].transpose(1, 0, 2, 3).reshape(74, 3, 40)[::2]
    _check_attention(held, table, lengths, [xs[:20], xs[20:]], [p[:20].float().cpu().numpy(), p[20:].float().cpu().numpy()], dtype, 40)


def test_offsets_past_32_bits(dgq):
    """Blocks on both sides of 2 GiB and 4 GiB of codes."""
    import torch
    S, H, d = 128, 8, 256
    per = H * S * 2 * d                                     # 512 KiB a block
    n_blocks = (4 << 30) // per + 40
    c = dgq.KVCache.empty(n_blocks, S, H, d)
    rng = np.random.default_rng(17)
    ids = [3, (2 << 30) // per - 1, (2 << 30) // per, (4 << 30) // per - 1, (4 << 30) // per, n_blocks - 1]
    n = 6 * S - 9
    k, kn = _floats(rng, (n, H, d), "bf16")
    v, vn = _floats(rng, (n, H, d), "bf16")
    dgq.dgq_kv_store(c, k, v, _i32([(b, i * S, 0, min(S, n - i * S)) for i, b in enumerate(ids)]))
    table = _i32([ids])
    k2, v2 = dgq.dgq_kv_load(c, table, _i32([n]), n)
    torch.cuda.synchronize()
    for x, y in ((k2[0].cpu().numpy(), kn), (v2[0].cpu().numpy(), vn)):
        for i in range(6):
            rows = slice(i * S, min(n, i * S + S))
            lim = np.abs(y[rows]).max((0, 2)) / 127 * 0.5001
            assert (np.abs(x[rows] - y[rows]).max((0, 2)) <= lim).all()
    for N in (1, 40, 4200):
        q, qn = _floats(rng, (1, N, H, d), "fp32")
        out = dgq.dgq_xattn_kv(q, c, table, _i32([n])).cpu().numpy()
        k64, v64 = k2[0].cpu().numpy().astype(np.float64), v2[0].cpu().numpy().astype(np.float64)
        want, big = ref.attention(qn[0].astype(np.float64), k64, v64)
        # (the values read back carry one more rounding, 2^-24 of K and V)
        assert (np.abs(out[0] - want) <= ref.tolerance("fp32", d, n, big * 1.5, v64, want) + 2.0 ** -23 * np.abs(v64).max()).all()


# ---- together ------------------------------------------------------------------------------------------------------------

def test_requests_come_and_go(dgq):
    """Several steps of a server: prompts arrive in pieces of 77 rows, are attended to, finish, and their blocks go to
    others; the lists never leave the device."""
    import torch
    rng = np.random.default_rng(20)
    S, H, G, d, B, W = 32, 2, 2, 40, 6, 8
    n_blocks = 30
    c = _cache(dgq, n_blocks, S, H, d)
    mirror = _read(c)
    table = np.full((B, W), -1)
    lengths, free = [0] * B, list(rng.permutation(n_blocks))
    d_len, d_free, d_n, d_table = _i32(lengths), _i32(free), _i32([n_blocks]), _i32(table)
    for step in range(7):
        done = (rng.random(B) < 0.3).astype(np.uint8)
        new = rng.choice([0, 1, 77, 77, 20], B)
        d_len, d_n = dgq.dgq_kv_release(torch.from_numpy(done).cuda(), d_len, d_table, d_free, d_n, S)
        free, lengths = ref.release(done, lengths, table, free, len(free), S)
        rows = int(new.sum())
        plan = dgq.dgq_kv_plan(d_len, _i32(new), d_table, d_free, d_n, S, rows)
        d_len, d_n = plan.lengths, plan.n_free
        table, lengths, n_free, offsets, runs, counts = ref.plan(lengths, new, table, free, len(free), S, rows)
        free = free[:n_free]
        kv, kvn = _floats(rng, (max(rows, 1), 2, H, d), "fp16")
        dgq.dgq_kv_store(c, kv[:, 0], kv[:, 1], plan.runs)
        ref.store(mirror, kvn[:, 0], kvn[:, 1], runs)
        q, qn = _floats(rng, (B, 21, H * G, d), "fp16")
        out = dgq.dgq_xattn_kv(q, c, d_table, d_len)
        torch.cuda.synchronize()
        assert d_len.tolist() == [int(x) for x in lengths] and d_n.tolist() == [n_free] and plan.counts.tolist() == counts
        assert d_free[:n_free].tolist() == [int(x) for x in free]
        _same_cache(_read(c), mirror, [r[0] for r in runs])
        _check_attention(mirror, table, lengths, qn, out.float().cpu().numpy(), "fp16", d)
        k, v = dgq.dgq_kv_load(c, d_table, d_len, 80, dtype=torch.float16)
        for b, n in enumerate(lengths):
            for r in range(min(n, 80)):
                assert np.array_equal(k[b, r].cpu().numpy(), mirror.values(0, table[b, r // S], r % S).astype(np.float16))


def test_load_feeds_the_log2_attention(dgq):
    """The values of one prompt length, read back, are the k and v of dgq_xattn_logq; its product with one key's weight
    near 1 is that key's value."""
    import torch
    rng = np.random.default_rng(21)
    c, table, held = _filled(dgq, rng, [77, 77], 32, 2, 40)
    k, v = dgq.dgq_kv_load(c, _i32(table), _i32([77, 77]), 77)
    bias = torch.zeros(77, device="cuda")
    bias[0] = 60.0
    q, _ = _floats(rng, (2, 50, 2, 40), "fp32")
    out, _ = dgq.dgq_xattn_logq(q, k, v, bias, 8)
    torch.cuda.synchronize()
    assert torch.allclose(out, v[:, :1].expand_as(out), rtol=0, atol=1e-5 * float(v.abs().max()))


def test_two_prompts_share_blocks(dgq):
    import torch
    rng = np.random.default_rng(22)
    c, table, held = _filled(dgq, rng, [77, 100], 32, 2, 40)
    both = np.stack([table[0], table[1], table[0], table[0]])
    q, qn = _floats(rng, (4, 19, 2, 40), "bf16")
    out = dgq.dgq_xattn_kv(q, c, _i32(both), _i32([77, 100, 77, 40])).float().cpu().numpy()
    _check_attention(held, both, [77, 100, 77, 40], qn, out, "bf16", 40)


@pytest.mark.parametrize("N", [50, 1])
def test_captured_step(dgq, N):
    """Release, plan, store and attention in one graph whose inputs change between replays; every replay gives the eager
    result, and two graphs with a workspace each do not disturb one another."""
    import torch
    S, H, d, B, W, rows = 32, 2, 64, 3, 40, 120
    nbytes = dgq.dgq_xattn_kv_workspace_bytes(B, N, False, H, H, d, W, S)

    def make(seed):
        rng = np.random.default_rng(seed)
        c = _cache(dgq, 90, S, H, d)
        t = dict(done=torch.zeros(B, dtype=torch.uint8, device="cuda"), lengths=_i32([0] * B), new=_i32([0] * B),
                 table=_i32(np.full((B, W), -1)), free=_i32(rng.permutation(90)), n_free=_i32([90]), mid=_i32([0] * B),
                 mid_n=_i32([0]), out_n=_i32([0]), out_len=_i32([0] * B), offsets=_i32([0] * (B + 1)), counts=_i32([0] * 4),
                 runs=_i32(np.zeros((rows // S + 2 * B, 4))), k=torch.zeros(rows, H, d, device="cuda"),
                 v=torch.zeros(rows, H, d, device="cuda"), q=torch.zeros(B, N, H, d, device="cuda"),
                 out=torch.zeros(B, N, H, d, device="cuda"), ws=torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda"))
        return c, t, rng

    def step(c, t):
        dgq.dgq_kv_release(t["done"], t["lengths"], t["table"], t["free"], t["n_free"], S, lengths_out=t["mid"], n_free_out=t["mid_n"])
        dgq.dgq_kv_plan(t["mid"], t["new"], t["table"], t["free"], t["mid_n"], S, rows, lengths_out=t["out_len"],
                        n_free_out=t["out_n"], row_offsets=t["offsets"], runs=t["runs"], counts=t["counts"])
        dgq.dgq_kv_store(c, t["k"], t["v"], t["runs"])
        dgq.dgq_xattn_kv(t["q"], c, t["table"], t["out_len"], out=t["out"], workspace=t["ws"])
        t["lengths"].copy_(t["out_len"])
        t["n_free"].copy_(t["out_n"])

    def feed(t, rng):
        t["done"].copy_(torch.from_numpy((rng.random(B) < 0.2).astype(np.uint8)))
        t["new"].copy_(_i32(rng.choice([0, 1, 20, 40], B)))
        for n in "kvq":
            t[n].copy_(torch.from_numpy(rng.standard_normal(t[n].shape).astype(np.float32)))

    eager, graphs = [make(1), make(2)], []
    captured = [make(1), make(2)]
    for c, t, _ in captured:
        fresh = {n: x.clone() for n, x in t.items()}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(c, t)  # warm-up
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step(c, t)
        torch.cuda.synchronize()
        for n, x in fresh.items():
            t[n].copy_(x)
        graphs.append(g)
    for rep in range(5):
        for (ec, et, er), (cc, ct, cr) in zip(eager, captured):
            feed(et, er)
            feed(ct, cr)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        for ec, et, _ in eager:
            step(ec, et)
        torch.cuda.synchronize()
        for (ec, et, _), (cc, ct, _) in zip(eager, captured):
            for n in ("out", "lengths", "n_free", "table", "runs", "counts", "offsets"):
                assert torch.equal(et[n], ct[n]), (rep, n)
            assert torch.isfinite(et["out"]).all()
    assert int(eager[0][1]["lengths"].max()) > 0


def test_on_another_stream(dgq):
    import torch
    rng = np.random.default_rng(23)
    lengths = [1500, 900]
    c, table, held = _filled(dgq, rng, lengths, 64, 2, 64)
    q, qn = _floats(rng, (2, 2, 2, 64), "fp32")
    t, n = _i32(table), _i32(lengths)
    want = dgq.dgq_xattn_kv(q, c, t, n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [dgq.dgq_xattn_kv(q, c, t, n, stream=side) for _ in range(20)]  # workspaces dropped at once
    with torch.cuda.stream(side):
        got.append(dgq.dgq_xattn_kv(q, c, t, n))
    torch.cuda.synchronize()
    assert torch.cuda.current_stream() != side
    assert all(torch.equal(x, want) for x in got)


# ---- refusals --------------------------------------------------------------------------------------------------------------

def test_refusals(dgq):
    import torch
    c, table, _ = _filled(dgq, np.random.default_rng(1), [40, 50], 32, 2, 16)
    t, n = _i32(table), _i32([40, 50])
    q = torch.zeros(2, 5, 2, 16, device="cuda")
    k = torch.zeros(9, 2, 16, device="cuda")
    runs = _i32([(0, 0, 0, 9)])
    E, V, T = dgq.DgqError, ValueError, TypeError

    def refused(error, call, *args, code=None, **kw):
        with pytest.raises(error) as e:
            call(*args, **kw)
        assert code is None or e.value.code == code

    x = dgq.dgq_xattn_kv
    refused(T, x, q.double(), c, t, n)
    refused(T, x, q.cpu(), c, t, n)
    refused(T, x, q, c, t.long(), n)
    refused(V, x, q[0], c, t, n)                                            # packed queries without offsets
    refused(V, x, q[0], c, t, n, q_offsets=_i32([0, 5]))
    refused(V, x, q[:1], c, t, n)
    refused(V, x, torch.zeros(2, 5, 2, 24, device="cuda"), c, t, n)
    refused(V, x, q, c, t, _i32([40]))
    refused(V, x, q, c, t, n, out=torch.zeros(2, 5, 2, 16, device="cuda", dtype=torch.float16))
    refused(V, x, q, c, t, n, out=torch.zeros(2, 5, 1, 16, device="cuda"))
    refused(E, x, torch.zeros(2, 5, 3, 16, device="cuda"), c, t, n, code=-4)  # 3 query heads to 2
    refused(T, x, torch.zeros(2, 5, 2, 32, device="cuda")[..., ::2], c, t, n)
    refused(E, x, torch.zeros(2, 5, 2, 18, device="cuda")[..., :16], c, t, n, code=-2)
    refused(E, x, torch.zeros(2 * 5 * 2 * 16 + 1, device="cuda")[1:].view(2, 5, 2, 16), c, t, n, code=-2)
    refused(V, x, q, dgq.KVCache(c.data[:-1], c.n_blocks, 32, 2, 16), t, n)
    refused(E, x, q, dgq.KVCache(c.data, c.n_blocks, 48, 2, 16), t, n, code=-4)
    few = torch.zeros(2, 1, 2, 16, device="cuda")
    wide = _i32(np.tile(table, (1, 20)))
    need = dgq.dgq_xattn_kv_workspace_bytes(2, 1, False, 2, 2, 16, wide.shape[1], 32)
    assert need > 0
    refused(E, x, few, c, wide, n, workspace=torch.empty(need - 16, dtype=torch.uint8, device="cuda"), code=-6)

    s = dgq.dgq_kv_store
    refused(V, s, c, k, k.half(), runs)
    refused(V, s, c, k, k[:5], runs)
    refused(V, s, c, k[:, :1], k[:, :1], runs)
    refused(V, s, c, k, k, runs[0])
    refused(T, s, c, k, k, runs.long())
    refused(E, s, c, torch.zeros(9, 2, 18, device="cuda")[..., :16], k, runs, code=-2)

    refused(V, dgq.dgq_kv_load, c, t, n, -1)
    refused(V, dgq.dgq_kv_load, c, t, n, 9, dtype=torch.float64)
    refused(T, dgq.dgq_kv_load, c, t, n, 9, dtype="fp32")
    refused(V, dgq.dgq_kv_load, c, t, n, 9, k=torch.zeros(2, 8, 2, 16, device="cuda"))
    refused(V, dgq.dgq_kv_load, c, t, _i32([1]), 9)

    free, nf, new = _i32(np.arange(9)), _i32([9]), _i32([3, 4])
    p = dgq.dgq_kv_plan
    refused(V, p, n, _i32([3]), t, free, nf, 32, 7)
    refused(V, p, n, new, t, free, _i32([9, 9]), 32, 7)
    refused(E, p, n, new, t, free, nf, 48, 7, code=-4)
    refused(E, p, n, new, t, free, nf, 32, -1, code=-1)
    refused(E, p, n, new, t, free, nf, 32, 7, lengths_out=n, code=-1)
    refused(E, p, n, new, t, free, nf, 32, 7, lengths_out=new, code=-1)
    refused(E, p, n, new, t, free, nf, 32, 7, n_free_out=nf, code=-1)
    refused(E, p, n, new, t, free, nf, 32, 100, runs=_i32(np.zeros((6, 4))), code=-3)
    refused(V, p, n, new, t, free, nf, 32, 7, runs=_i32(np.zeros(16)))
    many = _i32(np.zeros(4097))
    refused(E, p, many, many, _i32(np.zeros((4097, 1))), free, nf, 32, 7, code=-4)
    done = torch.zeros(2, dtype=torch.uint8, device="cuda")
    refused(V, dgq.dgq_kv_release, done[:1], n, t, free, nf, 32)
    refused(E, dgq.dgq_kv_release, done, n, t, free, nf, 32, lengths_out=n, code=-1)
    refused(V, dgq.KVCache.empty, 4, 32, 2, 20)
    torch.cuda.synchronize()
