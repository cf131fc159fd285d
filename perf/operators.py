"""The calls around the 8-bit cache of text keys and values, as timed cases, with their plain forms.

A prompt's keys and values do not change over the denoising steps, so a server writes them once, in 8 bits, into blocks
of a cache that all its requests share, and every step's cross-attention reads them from there.  Three kinds of case:

  plan   one scheduling step: finished requests give their blocks back (dgq_kv_release), the others' new rows get
         blocks and the runs that say which rows go where (dgq_kv_plan).  Whole numbers only.
  store  rows of K and V go into the cache (dgq_kv_store: one scale per block and head, for K and for V), and the
         requests' whole rows come back as the values the cache holds (dgq_kv_load)
  attn   cross-attention of each request's queries to its own rows of the cache (dgq_xattn_kv)

The cache's bytes (all sizes in slots of a block of S, heads H, head width d, e = d rounded up to a multiple of 16):
codes u8 [blocks, H, S/32, 64 e], of each 32 slots first K as [e/16, 32 slots, 16 dims], then V as [e, 2, 16 slots],
where place i of half h is slot 4 h + i%4 + 8 ((i/4)%2) + 16 (i/8); a byte is the code + 128.  Behind the codes the
scales fp32 [blocks, H, 2] (K, V).

`own` False computes everything with elementary torch operations in fp32; True makes the package's calls.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
TEXT = 77  # rows of one prompt piece


def _plan(name, B, W, S, new, before, done):
    return dict(name=name, kind="plan", B=B, W=W, S=S, new=new, before=before, done=done)


def _store(name, B, H, d, S, dtype, before, low, high):
    return dict(name=name, kind="store", B=B, H=H, d=d, S=S, dtype=dtype, before=before, low=low, high=high)


def _attn(name, B, N, H, G, d, S, dtype, low, high, packed=False, shared=False):
    return dict(name=name, kind="attn", B=B, N=N, H=H, G=G, d=d, S=S, dtype=dtype, low=low, high=high, packed=packed,
                shared=shared)


def listed():
    return [
        # sixteen requests, a third of them finished, the rest take one more 77-token piece: a small server's step
        _plan("plan_16", 16, 8, 32, TEXT, 160, 3),
        # a large server: ragged prompts of up to 512 rows, one request in seven finished
        _plan("plan_2048", 2048, 24, 64, 512, 900, 7),
        # a prompt and the unconditional one at the 64 x 64 level of the smaller network: the least a store is called for
        _store("store_2x77x8x40", 2, 8, 40, 32, "fp32", 0, TEXT, TEXT),
        # the second and third pieces of long prompts, appended in the middle of blocks that are rescaled
        _store("store_16x77x20x64_append", 16, 20, 64, 64, "bf16", 154, 1, TEXT),
        # a batch of long prompts of a wide text encoder
        _store("store_64x512x16x128", 64, 16, 128, 128, "fp16", 0, 300, 512),
        # the 8 x 8 level of the smaller network, one prompt length: the smallest attention of a step, launch-bound
        _attn("attn_2x64x8x160", 2, 64, 8, 1, 160, 32, "fp32", TEXT, TEXT),
        # its 64 x 64 level, one prompt in one piece and one in two
        _attn("attn_2x4096x8x40", 2, 4096, 8, 1, 40, 32, "fp32", TEXT, 2 * TEXT),
        # the 64 x 64 level at batch 16, 10 heads of 64, prompts from one token to three pieces
        _attn("attn_16x4096x10x64", 16, 4096, 10, 1, 64, 32, "fp32", 1, 3 * TEXT),
        # the 32 x 32 level, images of different sizes packed one behind another, half of the batch on one shared prompt
        _attn("attn_8x1024x20x64_packed", 8, 1024, 20, 1, 64, 64, "fp16", 256, 512, packed=True, shared=True),
        # one query for each of 32 requests, four query heads to a cached one, states from one row to 8192: no matrix
        # work to speak of, the cache's bytes
        _attn("attn_32x1x32x128_single", 32, 1, 8, 4, 128, 64, "bf16", 1, 8192),
        # one query of one request over a long state: only a split over the rows fills the chip
        _attn("attn_1x1x8x64_single", 1, 1, 8, 1, 64, 32, "fp32", 32768, 32768),
        # the largest: 4096 queries to some 4000 rows, 24 heads of 128
        _attn("attn_2x4096x24x128", 2, 4096, 24, 1, 128, 128, "bf16", 3900, 4096),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["plan", "store", "attn", "attn", "attn"])
    S = rng.choice([32, 64, 128])
    if kind == "plan":
        new, before = _log(rng, 1, 600), _log(rng, 1, 900)
        c = _plan(None, _log(rng, 1, 2048), -(-(new + before) // S) + rng.randrange(3), S, new, before, rng.randrange(2, 9))
    elif kind == "store":
        d, high = 8 * rng.randrange(1, 25), _log(rng, 1, 512)
        before = rng.choice([0, _log(rng, 1, 300)])
        H = rng.randrange(1, 25)
        dtype = rng.choice(sorted(TYPES))
        most = max(1, 2 * 64 * 512 * 16 * 128 // ((high + before) * H * d * SIZE[dtype]))
        c = _store(None, _log(rng, 1, min(64, most)), H, d, S, dtype, before, rng.randrange(1, high + 1), high)
    else:
        single = rng.random() < 0.3
        dtype, d, G = rng.choice(sorted(TYPES)), 8 * rng.randrange(1, 25), rng.choice([1, 1, 2, 4, 7])
        H = rng.randrange(1, 1 + 24 // G)
        if single:
            N, high = rng.choice([1, 1, 1, 2, 3, 5]), _log(rng, 1, 32768)
            B = _log(rng, 1, max(1, min(64, (1 << 28) // (high * H * d))))
            packed = False
        else:
            N, high = _log(rng, 16, 4096), _log(rng, 1, 4096 if dtype != "fp32" else 1024)
            most = min(2e11 / (4.0 * N * high * H * G * d), 3e8 / (N * H * G * d * SIZE[dtype]), 4e8 / (N * H * G * high))
            B = _log(rng, 1, max(1, min(16, int(most))))
            packed = rng.random() < 0.3
        low = rng.choice([high, rng.randrange(0, high + 1)])
        c = _attn(None, B, N, H, G, d, S, dtype, low, high, packed=packed, shared=B > 1 and rng.random() < 0.3)
    del c["name"]
    return c


def _spread(low, high, n):
    """n whole numbers from low to high, the ends among them, in a mixed order."""
    if n == 1:
        return [high]
    step = next(s for s in (7, 5, 3, 11, 13, 1) if math.gcd(s, n) == 1)
    return [low + (high - low) * ((i * step + n - 1) % n) // (n - 1) for i in range(n)]


def _lengths(case):
    B, S = case["B"], case["S"]
    if case["kind"] == "attn":
        n = _spread(case["low"], case["high"], B)
        if case["shared"]:  # the second half of the batch reads request 0's rows
            n[(B + 1) // 2:] = [n[0]] * (B // 2)
        return n
    if case["kind"] == "store":
        return [case["before"] * (i + 1) // B for i in range(B)], _spread(case["low"], case["high"], B)
    before = _spread(0, case["before"], B)
    new = _spread(0, case["new"], B)[::-1]
    # a finished request's place in the batch is taken at a later step
    return before, [0 if i % case["done"] == 0 else min(n, case["W"] * S - b) for i, (b, n) in enumerate(zip(before, new))]


def _queries(case):
    """Queries of every request."""
    B, N = case["B"], case["N"]
    return _spread(max(1, N // 2), N, B) if case["packed"] else [N] * B


def _up(n, to):
    return -(-n // to)


def work(case):
    S = case["S"]
    if case["kind"] == "plan":
        before, new = _lengths(case)
        B, out = case["B"], [i % case["done"] == 0 for i in range(case["B"])]
        given = sum(_up(b, S) for b, o in zip(before, out) if o)
        left = [0 if o else b for b, o in zip(before, out)]
        taken = sum(_up(b + n, S) - _up(b, S) for b, n in zip(left, new))
        runs = sum(_up(b + n, S) - b // S for b, n in zip(left, new) if n)
        return {"bytes": 4.0 * (5 * B + 2 * given + 2 * taken + 4 * runs) + B, "flops": 0.0}
    if case["kind"] == "store":
        before, new = _lengths(case)
        H, d, size = case["H"], case["d"], SIZE[case["dtype"]]
        rows = sum(new)
        held = sum(b + n for b, n in zip(before, new))
        old = sum(b % S for b, n in zip(before, new) if n)  # rows in blocks that are rescaled: read and written
        room = case["B"] * max(b + n for b, n in zip(before, new))
        return {"bytes": 2.0 * H * d * (rows * size + rows + 2 * old + held + room * size), "flops": 4.0 * H * d * rows}
    lengths, n = _lengths(case), _queries(case)
    H, d = case["H"], case["d"]
    rows = sum(lengths[:(case["B"] + 1) // 2]) if case["shared"] else sum(lengths)
    return {"bytes": 2.0 * sum(n) * H * case["G"] * d * SIZE[case["dtype"]] + 2.0 * H * d * rows,
            "flops": 4.0 * H * case["G"] * d * sum(a * b for a, b in zip(n, lengths))}


# ---- the cache's bytes ---------------------------------------------------------------------------------------------

def _places(device):
    """slot of place (half, i) of a tile's 32"""
    h = torch.arange(2, device=device)[:, None]
    i = torch.arange(16, device=device)[None, :]
    return (4 * h + i % 4 + 8 * (i // 4 % 2) + 16 * (i // 8)).reshape(32)


def _pack(codes_k, codes_v):
    """codes i8 [n, S, H, d] -> bytes u8 [n, H, S/32, 64 e]"""
    n, S, H, d = codes_k.shape
    e, T = _up(d, 16) * 16, S // 32
    pad = lambda c: torch.nn.functional.pad(c.to(torch.int16) + 128, (0, e - d), value=128).to(torch.uint8)  # noqa: E731
    k = pad(codes_k).reshape(n, T, 32, H, e // 16, 16).permute(0, 3, 1, 4, 2, 5).reshape(n, H, T, 32 * e)
    v = pad(codes_v).reshape(n, T, 32, H, e)[:, :, _places(codes_v.device)].permute(0, 3, 1, 4, 2).reshape(n, H, T, 32 * e)
    return torch.cat([k, v], -1)


def _unpack(data, S, H, d):
    """bytes u8 [n, H, S/32, 64 e] -> codes K, V as fp32 [n, H, S, d]"""
    n, e, T = data.shape[0], _up(d, 16) * 16, S // 32
    k = data[..., :32 * e].reshape(n, H, T, e // 16, 32, 16).permute(0, 1, 2, 4, 3, 5).reshape(n, H, S, e)[..., :d]
    back = torch.argsort(_places(data.device))
    v = data[..., 32 * e:].reshape(n, H, T, e, 32)[..., back].transpose(3, 4).reshape(n, H, S, e)[..., :d]
    return k.float() - 128, v.float() - 128


def _views(state):
    """the cache's two parts: codes u8 [blocks, H, S/32, 64 e], scales fp32 [blocks, H, 2]"""
    nb, S, H, d = state["blocks"], state["S"], state["H"], state["d"]
    n = nb * H * S * 2 * _up(d, 16) * 16
    return state["cache"][:n].view(nb, H, S // 32, -1), state["cache"][n:].view(torch.float32).view(nb, H, 2)


def _quantize(x, old_scale):
    """x fp32 [n, S, H, d], old_scale [n, H] -> codes, scale.  Rows that the block does not hold are zeros."""
    s = x.abs().amax((1, 3)) / 127
    s = torch.maximum(torch.where(s < 2.0 ** -96, 0.0, s), old_scale)
    inv = torch.where(s > 0, 1 / s, 0.0)
    return (x * inv[:, None, :, None]).round().clamp(-127, 127).to(torch.int8), s


# ---- inputs --------------------------------------------------------------------------------------------------------

def _states(g, shape, dtype, dev):
    """Keys or values of text tokens: channels of different size, a first token that stands out."""
    x = torch.randn(shape, generator=g, device=dev)
    x *= 0.5 + torch.rand(shape[-2:], generator=g, device=dev)
    return x.to(dtype)


def _table(case, lengths, dev, g, spare=0):
    """A block of its own, anywhere in the cache, for every S rows of every request; the free list behind."""
    S = case["S"]
    count = [_up(n, S) for n in lengths]
    total = sum(count)
    ids = torch.randperm(total + spare, generator=g, device=dev, dtype=torch.int32)
    W = case.get("W") or max(1, max(count) + (case["kind"] == "store") * _up(case["high"], S))
    first = torch.tensor([sum(count[:i]) for i in range(len(count))], device=dev)
    col = torch.arange(W, device=dev)
    has = col[None, :] < torch.tensor(count, device=dev)[:, None]
    at = torch.where(has, first[:, None] + col[None, :], 0)
    table = torch.full((len(count), W), -1, dtype=torch.int32, device=dev)
    if total:
        table = torch.where(has, ids[at], table)
    return table.contiguous(), ids[total:].contiguous(), total + spare


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    B, S = case["B"], case["S"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    state = dict(case=case, kind=case["kind"], S=S, B=B)
    if case["kind"] == "plan":
        before, new = _lengths(case)
        room = sum(_up(n, S) + 1 for n in new)
        table, spare, blocks = _table(case, before, dev, g, room)
        free = torch.zeros(blocks, dtype=torch.int32, device=dev)  # the list of the free blocks, at its first n_free places
        free[:room] = spare
        rows = sum(new)
        done = (torch.arange(B, device=dev) % case["done"] == 0).to(torch.uint8)
        return state | dict(lengths=i32(before), new=i32(new), done=done,
                            table=table, free=free, n_free=i32([room]), rows=rows, max_runs=rows // S + 2 * B)
    H, d, dtype = case["H"], case["d"], TYPES[case["dtype"]]
    e = _up(d, 16) * 16
    state |= dict(H=H, d=d, dtype=dtype)
    before, new = _lengths(case) if case["kind"] == "store" else (_lengths(case), None)
    if case["kind"] == "attn":
        held = list(before)
        if case["shared"]:
            held[(B + 1) // 2:] = [0] * (B // 2)
        table, _, blocks = _table(case, held, dev, g, 1)
        if case["shared"]:
            table[(B + 1) // 2:] = table[0]
    else:
        table, free, blocks = _table(case, before, dev, g, 1 + sum(_up(b + n, S) - _up(b, S) for b, n in zip(before, new)))
    state |= dict(blocks=blocks, table=table, lengths=i32(before),
                  cache=torch.full((blocks * H * (S * 2 * e + 8),), 128, dtype=torch.uint8, device=dev))
    codes, scales = _views(state)
    live = torch.unique(table[table >= 0]).long()
    for at in live.split(max(1, (1 << 26) // (S * H * d))):  # what the requests wrote before
        k, v = (_states(g, (at.numel(), S, H, d), torch.float32, dev) for _ in range(2))
        none = torch.zeros(at.numel(), H, device=dev)
        (ck, sk), (cv, sv) = _quantize(k, none), _quantize(v, none)
        codes[at], scales[at] = _pack(ck, cv), torch.stack([sk, sv], -1)
    if case["kind"] == "store":
        total = [b + n for b, n in zip(before, new)]
        rows = sum(new)
        kv = _states(g, (rows, 2, H, d), dtype, dev)  # one projection's output: K and V are views of it
        lists = _plan_plain(state["lengths"], i32(new), table, free, i32([free.numel()]), S, rows, rows // S + 2 * B)
        n_runs = sum(_up(t, S) - b // S for b, t in zip(before, total))
        return state | dict(k=kv[:, 0], v=kv[:, 1], runs=lists["runs"], n_runs=n_runs,
                            room=max(total), table=lists["table"].contiguous(), lengths=lists["lengths"])
    n = _queries(case)
    rows = sum(n)
    q = torch.randn((rows, H * case["G"], d), generator=g, device=dev).mul_(2.0).to(dtype)
    offsets = i32([sum(n[:i]) for i in range(B + 1)]) if case["packed"] else None
    q = q if case["packed"] else q.view(B, case["N"], H * case["G"], d)
    return state | dict(q=q, offsets=offsets, G=case["G"], most=max(n))


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _release_plain(done, lengths, table, free, n_free, S):
    W = table.shape[1]
    count = torch.where(done != 0, (lengths.clamp(min=0).long() + S - 1) // S, 0).clamp(max=W)
    has = torch.arange(W, device=table.device)[None, :] < count[:, None]
    # requests in order, each one's blocks in order; what is not given back goes to a place behind the list
    to = n_free.long() + (count.cumsum(0) - count)[:, None] + torch.arange(W, device=table.device)[None, :]
    to = torch.where(has, to, free.numel())
    free.copy_(torch.cat([free, free[:1]]).scatter_(0, to.view(-1), table.view(-1))[:-1])
    return torch.where(done != 0, 0, lengths).to(torch.int32), n_free + count.sum().to(torch.int32)


def _plan_plain(lengths, new, table, free, n_free, S, rows, max_runs):
    B, W = table.shape
    old, add = lengths.long(), new.long()
    ends = add.clamp(min=0).cumsum(0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    total = old + add
    have, need = (old + S - 1) // S, (total + S - 1) // S
    ok = (old >= 0) & (add >= 0) & (total <= W * S) & (ends <= rows)
    take = torch.where(ok, need - have, 0)
    served = ok & ((add == 0) | (take.cumsum(0) <= n_free))
    take = torch.where(served, take, 0)
    first = take.cumsum(0) - take
    count = torch.where(served & (add > 0), need - old // S, 0)
    last = count.cumsum(0)
    i = torch.arange(max_runs, device=table.device)
    r = torch.searchsorted(last, i, right=True).clamp(max=B - 1)
    here = i < last[-1]
    j = i - (last[r] - count[r])
    col = old[r] // S + j
    slot = torch.where(j == 0, old[r] % S, 0)
    n = torch.minimum((col + 1) * S, total[r]) - col * S - slot
    fresh = here & (col >= have[r])
    pop = (n_free.long() - 1 - (first[r] + col - have[r])).clamp(0, free.numel() - 1)
    block = torch.where(fresh, free[pop], table[r, col.clamp(0, W - 1)])
    row = offsets[r] + col * S + slot - old[r]
    runs = torch.where(here[:, None], torch.stack([block.long(), row, slot, n], 1),
                       torch.tensor([-1, 0, 0, 0], device=table.device)).to(torch.int32)
    to = torch.where(fresh, r * W + col, B * W)
    table = torch.cat([table.view(-1), table.view(-1)[:1]]).scatter_(0, to, block)[:-1].view(B, W)
    counts = torch.stack([last[-1], take.sum(), (~served).sum(), offsets[-1]]).to(torch.int32)
    return dict(table=table, lengths=torch.where(served, total, old).to(torch.int32),
                n_free=(n_free - take.sum()).to(torch.int32), offsets=offsets.to(torch.int32), runs=runs, counts=counts)


def _store_plain(state):
    S, H, d = state["S"], state["H"], state["d"]
    codes, scales = _views(state)
    runs = state["runs"][:state["n_runs"]].long()
    block, row, slot, n = runs.unbind(1)
    at = torch.arange(S, device=block.device)[None, :]
    is_new = (at >= slot[:, None]) & (at < (slot + n)[:, None])
    is_old = (at < slot[:, None])
    src = torch.where(is_new, row[:, None] + at - slot[:, None], 0)
    held = _unpack(codes[block], S, H, d)
    packed, kept = [], []
    for x, c, s in zip((state["k"], state["v"]), held, scales[block].unbind(-1)):
        s = torch.where((slot > 0)[:, None], s, 0.0)
        x = torch.where(is_new[:, :, None, None], x[src].float(), 0.0)
        _, scale = _quantize(x, s)
        x = torch.where(is_old[:, :, None, None], c.transpose(1, 2) * s[:, None, :, None], x)
        inv = torch.where(scale > 0, 1 / scale, 0.0)
        packed.append((x * inv[:, None, :, None]).round().clamp(-127, 127).to(torch.int8))
        kept.append(scale)
    codes[block], scales[block] = _pack(*packed), torch.stack(kept, -1)


def _rows_plain(state, L):
    """The values that the requests' rows stand for: K, V as fp32 [B, H, L, d], L a multiple of S."""
    S, H, d = state["S"], state["H"], state["d"]
    codes, scales = _views(state)
    at = state["table"][:, :L // S].clamp(min=0).long()
    s = scales[at]  # [B, L/S, H, 2]
    for x, i in zip(_unpack(codes[at.reshape(-1)], S, H, d), (0, 1)):
        x = x.view(*at.shape, H, S, d) * s[..., i, None, None]
        yield x.transpose(1, 2).reshape(at.shape[0], H, L, d)


def _load_plain(state):
    L, S = state["room"], state["S"]
    has = torch.arange(L, device=state["table"].device)[None, :] < state["lengths"][:, None]
    return [torch.where(has[:, :, None, None], x[:, :, :L].transpose(1, 2), 0.0).to(state["dtype"])
            for x in _rows_plain(state, _up(L, S) * S)]


def _attn_plain(state):
    q, S, H, G, d = state["q"], state["S"], state["H"], state["G"], state["d"]
    B, offsets = state["B"], state["offsets"]
    W = state["table"].shape[1]
    if offsets is not None:  # packed queries, padded to the longest
        at = offsets[:-1, None].long() + torch.arange(state["most"], device=q.device)[None, :]
        owner = torch.repeat_interleave(torch.arange(B, device=q.device), offsets[1:] - offsets[:-1], output_size=q.shape[0])
        place = torch.arange(q.shape[0], device=q.device) - offsets[owner]
        q = q[at.clamp(max=q.shape[0] - 1)]
    N = q.shape[1]
    q = q.float().view(B, N, H, G, d).permute(0, 2, 3, 1, 4).reshape(B * H, G * N, d)
    k, v = _rows_plain(state, W * S)
    kt = k.reshape(B * H, W * S, d).transpose(1, 2).contiguous()
    x = torch.bmm(q, kt).mul_(1 / math.sqrt(d)).view(B, H, G * N, W * S)
    there = torch.arange(W * S, device=q.device)[None, :] < state["lengths"][:, None]
    x.masked_fill_(~there[:, None, None, :], -math.inf)
    x -= x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    x.exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.bmm(x.view(B * H, G * N, W * S), v.reshape(B * H, W * S, d)).view(B, H, G * N, d)
    out = torch.where(total > 0, out / total, 0.0)
    out = out.view(B, H, G, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, H * G, d).to(state["dtype"])
    return out if offsets is None else out[owner, place]


def run(state):
    kind, S = state["kind"], state["S"]
    if kind == "plan":
        if own:
            import paper_2501_04304_amd as dgq
            lengths, n_free = dgq.dgq_kv_release(state["done"], state["lengths"], state["table"], state["free"],
                                                 state["n_free"], S)
            p = dgq.dgq_kv_plan(lengths, state["new"], state["table"], state["free"], n_free, S, state["rows"])
            return dict(table=state["table"], lengths=p.lengths, n_free=p.n_free, offsets=p.row_offsets, runs=p.runs,
                        counts=p.counts, free=state["free"])
        lengths, n_free = _release_plain(state["done"], state["lengths"], state["table"], state["free"], state["n_free"], S)
        p = _plan_plain(lengths, state["new"], state["table"], state["free"], n_free, S, state["rows"], state["max_runs"])
        return p | dict(free=state["free"])
    if own:
        import paper_2501_04304_amd as dgq
        cache = dgq.KVCache(state["cache"], state["blocks"], S, state["H"], state["d"])
        if kind == "store":
            dgq.dgq_kv_store(cache, state["k"], state["v"], state["runs"])
            return list(dgq.dgq_kv_load(cache, state["table"], state["lengths"], state["room"], dtype=state["dtype"]))
        return dgq.dgq_xattn_kv(state["q"], cache, state["table"], state["lengths"], q_offsets=state["offsets"])
    if kind == "store":
        _store_plain(state)
        return _load_plain(state)
    return _attn_plain(state)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def _decode(state, block, which):
    """One block's codes of K (0) or V (1), [H, S, d] in 64 bits, from the description of the bytes."""
    S, H, d = state["S"], state["H"], state["d"]
    e = (d + 15) // 16 * 16
    nbytes = S * 2 * e
    b = state["cache"][block * H * nbytes:(block + 1) * H * nbytes].view(H, S // 32, 2, 32 * e)[:, :, which].double() - 128
    if which == 0:
        return torch.cat([b[:, :, c * 512:(c + 1) * 512].reshape(H, S, 16) for c in range(e // 16)], -1)[..., :d]
    b = b.view(H, S // 32, e, 2, 2, 2, 4)  # dim, half, sixteen, eight, four
    return b.permute(0, 1, 4, 5, 3, 6, 2).reshape(H, S, e)[..., :d]


def _exact_rows(state, b, n, which):
    S, H = state["S"], state["H"]
    at = state["blocks"] * H * S * 2 * ((state["d"] + 15) // 16 * 16)
    scales = state["cache"][at:].view(torch.float32).view(state["blocks"], H, 2)
    ids = state["table"][b, :(n + S - 1) // S].tolist()
    return torch.cat([_decode(state, i, which) * scales[i, :, which].double()[:, None, None] for i in ids], 1)[:, :n]


def exact(case, seed):
    if case["kind"] == "plan":
        return None
    state = prepare(case, seed)
    lengths = state["lengths"].tolist()
    if case["kind"] == "attn":
        if sum(lengths) / case["S"] * 2 > 40000:
            return None
        n, G, out = _queries(case), state["G"], []
        q = state["q"].reshape(-1, state["H"], G, state["d"])
        for b in range(case["B"]):
            x = q[sum(n[:b]):sum(n[:b + 1])].double()
            if lengths[b] == 0:
                out.append(torch.zeros_like(x))
                continue
            k, v = (_exact_rows(state, b, lengths[b], w) for w in (0, 1))
            heads = []
            for h in range(state["H"]):
                p = torch.softmax(x[:, h].reshape(-1, state["d"]) @ k[h].T.contiguous() / math.sqrt(state["d"]), -1)
                heads.append((p @ v[h]).view(n[b], G, -1))
            out.append(torch.stack(heads, 1))
        return torch.cat(out).view(*state["q"].shape)
    # the codes' roundings are those of the fp32 operations that define them; the values they stand for are in 64 bits
    got = []
    S, H, d = state["S"], state["H"], state["d"]
    before, new = _lengths(case)
    for which, x in enumerate((state["k"].float(), state["v"].float())):
        y = torch.zeros(case["B"], state["room"], H, d, dtype=torch.float64, device=x.device)
        at = state["blocks"] * H * S * 2 * ((d + 15) // 16 * 16)
        scales = state["cache"][at:].view(torch.float32).view(state["blocks"], H, 2)[..., which]
        row = 0
        for b in range(case["B"]):
            if before[b]:
                y[b, :before[b]] = _exact_rows(state, b, before[b], which).transpose(0, 1)
            at, end = before[b], before[b] + new[b]
            while at < end:
                to = min(end, at // S * S + S)
                rows, lo = x[row:row + to - at], at // S * S
                s = rows.abs().amax((0, 2)) / 127
                s[s < 2.0 ** -96] = 0
                old = scales[int(state["table"][b, at // S])] if at > lo else torch.zeros_like(s)
                s = torch.maximum(s, old)
                inv = torch.where(s > 0, 1 / s, torch.zeros_like(s))[None, :, None]
                whole = torch.cat([y[b, lo:at].float(), rows])
                y[b, lo:to] = torch.clamp(torch.round(whole * inv), -127, 127).double() * s.double()[None, :, None]
                row += to - at
                at = to
        got.append(y)
    return got
