"""A residual block as a denoising step runs it: the projections of the time embedding with 4-bit weights, norm and SiLU,
convolution, embedding and norm and SiLU, convolution.  Every call is held to its own definition on the inputs it got."""
import numpy as np
import pytest

import norm_reference
import w4_reference
from support import assert_close_fp32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dgq():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2501_04304_amd as m
    m.lib()
    return m


def _up(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


B, H, W, C, O, G, EMB, GROUP = 2, 16, 32, 64, 96, 8, 320, 64


class Block:
    """Weights of a block, its calls, and what each was given and gave."""

    def __init__(self, dgq, modulated):
        rng = np.random.default_rng(1)
        f = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
        self.dgq, self.modulated = dgq, modulated
        self.wide = (2 if modulated else 1) * O
        self.proj, self.proj_bias = f(self.wide, EMB) * np.float32(EMB ** -0.5), np.float32(0.1) * f(self.wide)
        self.norms = [(f(C), f(C)), (f(O), f(O))]
        self.convs = [(np.float32(0.05) * f(O, 9 * C), f(O)), (np.float32(0.05) * f(O, 9 * O), f(O))]
        self.w4 = dgq.dgq_w4_pack(dgq.W4Weight.empty(self.wide, EMB, GROUP), _up(self.proj))
        self.d_proj_bias = _up(self.proj_bias)
        self.d_norms = [tuple(_up(a) for a in n) for n in self.norms]
        self.handles = None

    def calibrate(self, x, emb):
        """Group tables and weights of the convolutions, from the maps of one pass."""
        self.handles = [None, None]
        for i in range(2):
            m = self.step(x, emb, stop=i)
            g = self.dgq.dgq_calibrate_groups(m, 8, 64, 1)
            g9 = self.dgq.dgq_groups_for_conv3x3(g)
            w, b = self.convs[i]
            self.handles[i] = (g, g9, self.dgq.dgq_pack_weight(g9, _up(w), _up(b), 8))

    def conv(self, i, m):
        g, g9, w = self.handles[i]
        codes, cls = self.dgq.dgq_quantize_act_conv3x3(g, g9, m, B, H, W)
        return self.dgq.dgq_linear_conv3x3(g9, w, codes, cls, B, H, W)

    def step(self, x, emb, stop=None, seen=None):
        dgq = self.dgq
        p = dgq.dgq_w4_matvec(emb, self.w4, self.d_proj_bias, act=dgq.ACT_NONE)
        a = dgq.dgq_groupnorm(x.view(B, H * W, C), G, *self.d_norms[0], act=dgq.ACT_SILU).view(B * H * W, C)
        if stop == 0:
            return a
        h = self.conv(0, a)
        terms = dict(scale=p[:, :O], shift=p[:, O:]) if self.modulated else dict(add=p)
        c = dgq.dgq_groupnorm(h.view(B, H * W, O), G, *self.d_norms[1], act=dgq.ACT_SILU, **terms).view(B * H * W, O)
        if stop == 1:
            return c
        y = self.conv(1, c)
        if seen is not None:
            seen.update(p=p, a=a, h=h, c=c, y=y)
        return y

    def free(self):
        for g, g9, w in self.handles:
            w.free(), g9.free(), g.free()


@pytest.mark.parametrize("modulated", [False, True])
def test_residual_block(dgq, oracle, modulated):
    import torch
    rng = np.random.default_rng(2)
    xn = (rng.standard_normal((B * H * W, C)) * (0.5 + rng.random(C))).astype(np.float32)
    en = rng.standard_normal((B, EMB)).astype(np.float32)
    x, emb = _up(xn), _up(en)
    block = Block(dgq, modulated)
    block.calibrate(x, emb)
    seen = {}
    y = block.step(x, emb, seen=seen)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in seen.items()}
    starts, ends = [0, H * W], [H * W, 2 * H * W]

    def close(v, want, tol):
        assert (np.abs(v.astype(np.float64) - want) <= tol).all()

    codes, words = w4_reference.quantize(block.proj, GROUP)
    close(got["p"], *w4_reference.matvec(en, codes, words, GROUP, block.wide, block.proj_bias, pieces=2))
    close(got["a"], *norm_reference.groupnorm(xn, starts, ends, G, *block.norms[0], silu=True))
    p = got["p"]
    terms = dict(scale=p[:, :O], shift=p[:, O:]) if modulated else dict(add=p)
    close(got["c"], *norm_reference.groupnorm(got["h"], starts, ends, G, *block.norms[1], silu=True, **terms))
    for i, (src, dst) in enumerate((("a", "h"), ("c", "y"))):
        og9 = oracle.groups_for_conv3x3(oracle.calibrate(got[src], 8, 64, 1))
        oq = oracle.quantize_act(og9, oracle.im2col3x3(got[src], B, H, W))
        owq, osw = oracle.quantize_weight(block.convs[i][0], 8)
        want = oracle.linear(og9, oq["q"], oq["cls"], owq, osw, block.convs[i][1])
        assert_close_fp32(got[dst], want[0] if isinstance(want, tuple) else want, dst)

    # the step in a graph, with other embeddings and maps between the replays
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        block.step(x, emb)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            out = block.step(x, emb)
    torch.cuda.synchronize()
    for rep in range(4):
        emb.copy_(_up(en * (1 + rep)))
        x.copy_(_up(xn * (1 - 0.1 * rep)))
        want = block.step(x, emb)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), rep
    x.copy_(_up(xn)), emb.copy_(_up(en))
    assert torch.equal(block.step(x, emb), y)
    block.free()
