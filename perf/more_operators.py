"""What stands around a U-Net's 3 x 3 convolutions, as timed cases, with their plain forms.

A residual block normalises its map by groups of channels, applies SiLU, convolves, and shifts or scales the next map by a
projection of the time embedding: a product of as many rows as there are images, whose time is the weights' bytes.  Three
kinds of case:

  norm    group norm over [pixels, channels] rows with SiLU, the embedding added before it or scaling and shifting after it
          (dgq_groupnorm)
  pack    a layer's weights into 4 bits with a scale and a zero for every group of inputs, and back to values
          (dgq_w4_pack, dgq_w4_unpack)
  matvec  products of few rows with such weights, with bias and SiLU (dgq_w4_matvec)

Packed weights of O outputs and C inputs (R = ceil(O/16), T = ceil(C/128)): codes u8 [R, T, 4 q, 16 rows, 4 j, 4], where the
32-bit word of (row tile, t, q, row, j) holds inputs 128 t + 32 j + 8 q + i, i of 0 .. 7, in nibble i/2 for even i and
4 + (i-1)/2 for odd i.  Behind the codes int32 [R, T, 16, 128/group]: the bits of the fp32 scale, whose lowest four are the
group's zero.  A value is scale * (code - zero).

`own` False computes everything with elementary torch operations in fp32; True makes the package's calls.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
EPS = 1e-5


def _norm(name, B, N, C, G, dtype, out, silu=True, add=False, mod=False, packed=False):
    return dict(name=name, kind="norm", B=B, N=N, C=C, G=G, dtype=dtype, out=out, silu=silu, add=add, mod=mod, packed=packed)


def _pack(name, O, C, group, dtype):
    return dict(name=name, kind="pack", O=O, C=C, group=group, dtype=dtype)


def _matvec(name, M, C, O, group, dtype, out, silu=False, bias=True):
    return dict(name=name, kind="matvec", M=M, C=C, O=O, group=group, dtype=dtype, out=out, silu=silu, bias=bias)


def listed():
    return [
        # the 8 x 8 level at batch 2: the smallest map of a step, launch-bound
        _norm("norm_2x64x1280", 2, 64, 1280, 32, "fp32", "fp32"),
        # the 64 x 64 level of one guided prompt, behind the block's first convolution: the embedding is added
        _norm("norm_2x4096x320_add", 2, 4096, 320, 32, "fp32", "fp32", add=True),
        # the 64 x 64 level at batch 16, embedding as scale and shift
        _norm("norm_16x4096x640_scale_shift", 16, 4096, 640, 32, "fp32", "fp32", mod=True),
        # images of different sizes packed one behind another, one of them empty; fp32 rows for the quantizer
        _norm("norm_8x4096x960_packed", 8, 4096, 960, 32, "bf16", "fp32", add=True, packed=True),
        # the last level of an image decoder, 1024 x 1024 pixels: one image, long groups of few channels
        _norm("norm_1x1048576x128", 1, 1048576, 128, 32, "fp16", "fp16"),
        # a time embedding's first layer, as a program loads it
        _pack("pack_1280x320", 1280, 320, 32, "fp32"),
        # a wide text encoder's layer
        _pack("pack_8192x8192", 8192, 8192, 128, "bf16"),
        # the time embedding of one guided prompt: the smallest product, launch-bound
        _matvec("matvec_2x320x1280", 2, 320, 1280, 32, "fp32", "fp32", silu=True),
        # the projections of all residual blocks stacked into one layer, sixteen guided prompts
        _matvec("matvec_32x1280x16640", 32, 1280, 16640, 64, "fp32", "fp32"),
        # odd sizes in both directions: rows that no vector load fits, a group and a tile that end early
        _matvec("matvec_7x2051x1003", 7, 2051, 1003, 64, "fp16", "fp16", silu=True),
        # one token through a wide feed-forward layer
        _matvec("matvec_1x4096x16384", 1, 4096, 16384, 128, "bf16", "bf16", bias=False),
        # the largest: one token, weights of 121 MB
        _matvec("matvec_4x8192x28672", 4, 8192, 28672, 128, "bf16", "fp32"),
    ]


MOST_VALUES = 1048576 * 128  # of a map
MOST_WEIGHTS = 8192 * 28672


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "matvec", "matvec", "pack"])
    dtype = rng.choice(sorted(TYPES))
    out = rng.choice([dtype, "fp32"])
    if kind == "norm":
        G = rng.choice([1, 4, 8, 16, 30, 32, 32, 32])
        C = G * rng.randrange(1, 1 + 2560 // G)
        size = max(SIZE[dtype], SIZE[out]) / 2  # bytes bind: fp32 maps of half the values
        N = _log(rng, 1, min(65536, int(MOST_VALUES / size) // C))
        B = _log(rng, 1, max(1, min(32, int(MOST_VALUES / size) // (N * C))))
        c = _norm(None, B, N, C, G, dtype, out, silu=rng.random() < 0.7, add=rng.random() < 0.4, mod=rng.random() < 0.3,
                  packed=rng.random() < 0.3)
    elif kind == "pack":
        c = _pack(None, _log(rng, 1, 8192), _log(rng, 1, 8192), rng.choice([32, 64, 128]), dtype)
    else:
        O = _log(rng, 1, 28672)
        C = _log(rng, 1, min(28672, MOST_WEIGHTS // O))
        C = C if rng.random() < 0.5 else 32 * -(-C // 32)
        M = _log(rng, 1, 64)
        c = _matvec(None, M, C, min(O, MOST_WEIGHTS // C), rng.choice([32, 64, 128]), dtype, out, silu=rng.random() < 0.3,
                    bias=rng.random() < 0.5)
    del c["name"]
    return c


def _up(n, to):
    return -(-n // to)


def _rows(case):
    """Pixels of every image."""
    B, N = case["B"], case["N"]
    if not case["packed"] or B == 1:
        return [N] * B
    return [N - (N * ((5 * i + 1) % B)) // (B - 1) for i in range(B)]  # N down to none, in a mixed order


def work(case):
    if case["kind"] == "norm":
        values = sum(_rows(case)) * case["C"]
        tables = 4 * case["C"] * (2 + case["B"] * (case["add"] + 2 * case["mod"]))
        return dict(bytes=values * (SIZE[case["dtype"]] + SIZE[case["out"]]) + tables, flops=10 * values)
    weights = case["O"] * case["C"]
    held = weights / 2 + 4 * case["O"] * _up(case["C"], case["group"])
    if case["kind"] == "pack":
        return dict(bytes=2 * weights * SIZE[case["dtype"]] + 2 * held, flops=8 * weights)
    M = case["M"]
    return dict(bytes=held + M * case["C"] * SIZE[case["dtype"]] + M * case["O"] * SIZE[case["out"]] + 4 * case["O"] * case["bias"],
                flops=2.0 * M * weights)


# ---- the packed weights' bytes -------------------------------------------------------------------------------------

def _nbytes(O, C, group):
    return _up(O, 16) * _up(C, 128) * (1024 + 64 * (128 // group))


def _quantize(w, group):
    """fp32 [O, C] -> codes u8 [16 R, 128 T], words int32 [16 R, 128 T / group].  Rows and inputs that are not there are
    zeros."""
    O, C = w.shape
    w = torch.nn.functional.pad(w, (0, 128 * _up(C, 128) - C, 0, 16 * _up(O, 16) - O)).unflatten(1, (-1, group))
    lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
    s = (((hi - lo) * (1 / 15)).view(torch.int32) & -16).view(torch.float32)
    s = torch.where(s >= 2.0 ** -96, s, 0.0)
    inv = torch.where(s > 0, 1 / s, 0.0)
    zero = (-lo * inv).round_().clamp_(0, 15)
    codes = (w * inv[:, :, None]).round_().add_(zero[:, :, None]).clamp_(0, 15).to(torch.uint8)
    return codes.flatten(1), s.view(torch.int32) | zero.to(torch.int32)


def _lay_out(codes, words, group):
    rows, C = codes.shape
    c = codes.view(rows // 16, 16, C // 128, 4, 4, 4, 2)  # row tile, row, t, j, q, pair, which of the pair
    c = c.permute(0, 2, 4, 1, 3, 6, 5)  # row tile, t, q, row, j, nibbles in order
    c = c.reshape(rows // 16, C // 128, 4, 16, 4, 4, 2)
    c = (c[..., 0] | (c[..., 1] << 4)).contiguous()
    s = words.view(rows // 16, 16, C // 128, 128 // group).permute(0, 2, 1, 3).contiguous()
    return torch.cat([c.view(-1), s.view(-1).view(torch.uint8)])


def _values(data, O, C, group):
    """The packed weights as fp32 [O, C]."""
    R, T = _up(O, 16), _up(C, 128)
    n = R * T * 1024
    c = data[:n].view(R, T, 4, 16, 4, 4)
    c = torch.stack([c & 15, c >> 4], -1).view(R, T, 4, 16, 4, 2, 4)
    c = c.permute(0, 3, 1, 4, 2, 6, 5).reshape(16 * R, 128 * T // group, group)
    s = data[n:].view(torch.int32).view(R, T, 16, 128 // group).permute(0, 2, 1, 3).reshape(16 * R, -1)
    zero, s = (s & 15).float(), (s & -16).view(torch.float32)
    return ((c.float() - zero[:, :, None]) * s[:, :, None]).flatten(1)[:O, :C]


# ---- inputs --------------------------------------------------------------------------------------------------------

def _layer(g, O, C, dev):
    """A layer's weights: rows and inputs of different size."""
    w = torch.randn((O, C), generator=g, device=dev)
    w *= (0.5 + torch.rand((O, 1), generator=g, device=dev)) / math.sqrt(C)
    w *= 0.5 + torch.rand((1, C), generator=g, device=dev)
    return w


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    state = dict(case=case, kind=case["kind"], dtype=TYPES[case["dtype"]], out=TYPES[case.get("out", case["dtype"])])
    if case["kind"] == "norm":
        B, C, rows = case["B"], case["C"], _rows(case)
        # a convolution's output: channels of different mean and size
        x = normal(sum(rows), C).mul_(0.3 + 2 * torch.rand((C,), generator=g, device=dev)).add_(normal(C)).to(state["dtype"])
        state |= dict(weight=1 + 0.2 * normal(C), bias=0.2 * normal(C), add=None, scale=None, shift=None, offsets=None)
        # a block's columns of the stacked projections' output
        emb = 0.5 * normal(B, 3 * C)
        if case["add"]:
            state["add"] = emb[:, :C]
        if case["mod"]:
            state |= dict(scale=emb[:, C:2 * C], shift=emb[:, 2 * C:])
        if case["packed"]:
            state["offsets"] = torch.tensor([sum(rows[:i]) for i in range(B + 1)], dtype=torch.int32, device=dev)
        return state | dict(x=x if case["packed"] else x.view(B, case["N"], C))
    O, C, group = case["O"], case["C"], case["group"]
    w = _layer(g, O, C, dev)
    if case["kind"] == "pack":
        return state | dict(w=w.to(state["dtype"]), data=torch.empty(_nbytes(O, C, group), dtype=torch.uint8, device=dev))
    x = normal(case["M"], C)
    x *= torch.where(torch.rand((C,), generator=g, device=dev) < 0.01, 8.0, 1.0)  # some inputs stand out
    return state | dict(x=x.to(state["dtype"]), data=_lay_out(*_quantize(w, group), group),
                        bias=0.1 * normal(O) if case["bias"] else None)


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _silu(t):
    return t / (1 + torch.exp(-t))


def _norm_plain(state):
    case, x = state["case"], state["x"].float()
    G, C, offsets = case["G"], case["C"], state["offsets"]
    per = lambda t: t[:, None]  # noqa: E731  an image's row for all its pixels
    if offsets is not None:
        owner = torch.searchsorted(offsets[1:], torch.arange(x.shape[0], device=x.device, dtype=torch.int32), right=True)
        per = lambda t: t[owner]  # noqa: E731
    if state["add"] is not None:
        x = x + per(state["add"])
    x = x.unflatten(-1, (G, C // G))
    if offsets is None:
        mean = x.mean((1, 3), keepdim=True)
        x = x - mean
        rstd = 1 / torch.sqrt(x.square().mean((1, 3), keepdim=True) + EPS)
    else:
        n = (offsets[1:] - offsets[:-1]).clamp(min=1)[:, None] * (C // G)
        # the pixels' sums side by side, images in rows of their longest, zeros behind each one's own
        at = offsets[:-1, None] + torch.arange(case["N"], device=x.device, dtype=torch.int32)
        there = (at < offsets[1:, None])[..., None]
        at = at.clamp(max=x.shape[0] - 1)
        of = lambda t: torch.where(there, t.sum(2)[at], 0.0).sum(1, dtype=torch.float64) / n  # noqa: E731
        x = x - per(of(x).float())[..., None]
        rstd = per((1 / torch.sqrt(of(x.square()) + EPS)).float())[..., None]
    t = (x * rstd).flatten(-2) * state["weight"] + state["bias"]
    if state["scale"] is not None:
        t = t * (1 + per(state["scale"])) + per(state["shift"])
    return (_silu(t) if case["silu"] else t).to(state["out"])


def run(state):
    case, kind = state["case"], state["kind"]
    if own:
        import paper_2501_04304_amd as dgq
        if kind == "norm":
            return dgq.dgq_groupnorm(state["x"], case["G"], state["weight"], state["bias"], EPS,
                                     act=dgq.ACT_SILU if case["silu"] else dgq.ACT_NONE, add=state["add"], scale=state["scale"],
                                     shift=state["shift"], offsets=state["offsets"], dtype=state["out"])
        weight = dgq.W4Weight(state["data"], case["O"], case["C"], case["group"])
        if kind == "pack":
            dgq.dgq_w4_pack(weight, state["w"])
            return dgq.dgq_w4_unpack(weight, dtype=state["dtype"])
        return dgq.dgq_w4_matvec(state["x"], weight, state["bias"], act=dgq.ACT_SILU if case["silu"] else dgq.ACT_NONE,
                                 dtype=state["out"])
    if kind == "norm":
        return _norm_plain(state)
    O, C, group = case["O"], case["C"], case["group"]
    if kind == "pack":
        state["data"].copy_(_lay_out(*_quantize(state["w"].float(), group), group))
        return _values(state["data"], O, C, group).to(state["dtype"])
    y = state["x"].float() @ _values(state["data"], O, C, group).T
    if state["bias"] is not None:
        y = y + state["bias"]
    return (_silu(y) if case["silu"] else y).to(state["out"])


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "norm":
        G, C, got, at = case["G"], case["C"], [], 0
        x = state["x"].reshape(-1, C)
        for b, n in enumerate(_rows(case)):
            t = x[at:at + n].double()
            at += n
            if state["add"] is not None:
                t += state["add"][b].double()
            t = t.view(n, G, C // G)
            if n:
                var, mean = torch.var_mean(t, dim=(0, 2), correction=0)
                t = (t - mean[None, :, None]) / torch.sqrt(var + EPS)[None, :, None]
            t = torch.addcmul(state["bias"].double(), t.reshape(n, C), state["weight"].double())
            if state["scale"] is not None:
                t = torch.addcmul(t + state["shift"][b].double(), t, state["scale"][b].double())
            got.append(t * torch.sigmoid(t) if case["silu"] else t)
        return torch.cat(got).view(state["x"].shape)
    O, C, group = case["O"], case["C"], case["group"]
    if case["kind"] == "pack":
        # the codes' roundings are those of the fp32 operations that define them; the values they stand for are in 64 bits
        y = torch.empty(O, C, dtype=torch.float64, device=state["w"].device)
        for at in range(0, C, group):
            w = state["w"][:, at:at + group].float()
            low, high = torch.minimum(w.min(1).values, torch.zeros(())), torch.maximum(w.max(1).values, torch.zeros(()))
            bits = ((high - low) * torch.tensor(1 / 15, dtype=torch.float32)).view(torch.int32)
            s = (bits - bits % 16).view(torch.float32)
            s[s < 2.0 ** -96] = 0
            inv = torch.where(s > 0, 1 / s, s)
            zero = torch.round(-low * inv).clip(0, 15)[:, None]
            y[:, at:at + group] = (torch.clip(torch.round(w * inv[:, None]) + zero, 0, 15) - zero).double() * s[:, None].double()
        return y
    # every input's nibble by its place, one input of the 128 of a tile after another
    R, T = (O + 15) // 16, (C + 127) // 128
    words = state["data"][:R * T * 1024].view(torch.int32).view(R, T, 4, 16, 4)
    marks = state["data"][R * T * 1024:].view(torch.int32).view(R, T, 16, 128 // group)
    y = torch.zeros(case["M"], 16 * R, dtype=torch.float64, device=words.device)
    x = state["x"].double()
    for k in range(min(128, C)):
        j, q, i = k // 32, k // 8 % 4, k % 8
        code = (words[:, :, q, :, j] >> (4 * (i // 2 + 4 * (i % 2)))) % 16
        mark = marks[:, :, :, k // group]
        v = (mark - mark % 16).view(torch.float32).double() * (code - mark % 16).double()  # [R, T, 16]
        cols = x[:, k::128]
        v = v[:, :cols.shape[1]].permute(1, 0, 2).reshape(cols.shape[1], 16 * R)
        y += cols @ v
    y = y[:, :O]
    if state["bias"] is not None:
        y = y + state["bias"].double()
    return y * torch.sigmoid(y) if case["silu"] else y
