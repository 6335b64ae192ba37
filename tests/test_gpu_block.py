"""MultiViewBlock on slices of the views: norms, products, attention and the
feed-forward part together, against a plain float64 form of the same block, and
as the denoiser of the cached loop.

Tolerances: of the block's own roundings the ones that reach the output are
twelve (two norms, the projection, normed and turned heads, weights, attention's output, its
projection, the sum, the feed-forward part's middle and the output), each of at most half a step of its
value; gains, gates and norms keep the 2-norm within a factor of two of what
they get, so the output's relative error in the 2-norm is below 2 sqrt(12) half steps where they are independent
and below 24 in any case.  In 8 bits the plain form rounds the same operands the same way (a rounding at a
border may go either way: of half a step each, for few values), so the layer's own type decides there as well, with
twice as many roundings counted."""
import math

import pytest
import torch

from synth.configs import C2, C4

from conftest import latent_maps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACTS = {0: lambda p: p, 1: lambda p: p * torch.sigmoid(p), 2: lambda p: p * torch.special.erfc(-p / math.sqrt(2)) / 2}


def block_for(pos, dtype, gated=True, act=1, width=64, heads=4, kv_heads=2, dim=64, hidden=176, biases=True):
    from paper_2608_13255_amd.multiview import MultiViewBlock
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    block = MultiViewBlock(pos, width, heads, kv_heads, dim, hidden, act=act, gated=gated, dtype=dtype, generator=g)
    near_one = lambda n: 1 + 0.2 * torch.randn(n, generator=g, device=DEV)
    block.q_gain.copy_(near_one(dim)), block.k_gain.copy_(near_one(dim))
    block.attention_gain.copy_(near_one(width)), block.feed_gain.copy_(near_one(width))
    if biases:
        for name in ("qkv", "out", "in", "down"):
            setattr(block, "b_" + name, 0.1 * torch.randn(getattr(block, "w_" + name).shape[0], generator=g, device=DEV))
    return block


def eight(x):
    s = x.abs().amax(-1, keepdim=True).clamp_min(448 * 2.0 ** -126) / 448
    return (x / s).float().to(torch.float8_e4m3fn).double() * s


def plain(block, x, views, base=10000.0):
    """The block in float64: asset by asset, head by head."""
    B = x.shape[0]
    h, hk, D = block.heads, block.kv_heads, block.dim
    fg = block.foreground[:, list(views)].cpu()
    x = x.double().cpu()
    put = eight if block.eight_bits is not None else lambda t: t
    w = {n: put(getattr(block, "w_" + n).double().cpu()) for n in ("qkv", "out", "in", "down")}
    bias = {n: 0.0 if getattr(block, "b_" + n) is None else getattr(block, "b_" + n).double().cpu() for n in w}
    gain = {n: getattr(block, n).double().cpu() for n in ("q_gain", "k_gain", "attention_gain", "feed_gain")}
    freq = torch.cat([base ** (-torch.arange(m, dtype=torch.float64) / m) for m in block.sections])
    axis = torch.cat([torch.full((m,), a) for a, m in enumerate(block.sections)])
    rms = lambda u, g: u / (u.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g
    product = lambda u, n: put(u) @ w[n].t() + bias[n]
    y = torch.zeros_like(x)
    for b in range(B):
        at = fg[b].nonzero()
        t = x[b][fg[b]]
        q, k, v = product(rms(t, gain["attention_gain"]), "qkv").view(-1, h + 2 * hk, D).split([h, hk, hk], 1)
        place = torch.stack([torch.tensor(list(views))[at[:, 0]], at[:, 1], at[:, 2]], 1).double()
        angle = (place[:, axis] * freq)[:, None]
        c, s = angle.cos(), angle.sin()

        def turn(u, g):
            u = rms(u, g)
            p, r = u[..., :D // 2], u[..., D // 2:]
            return torch.cat([p * c - r * s, r * c + p * s], -1)

        q, k = turn(q, gain["q_gain"]), turn(k, gain["k_gain"])
        o = torch.stack([torch.softmax(q[:, i] @ k[:, i * hk // h].t() / math.sqrt(D), -1) @ v[:, i * hk // h]
                         for i in range(h)], 1)
        t = t + product(o.reshape(-1, h * D), "out")
        m = product(rms(t, gain["feed_gain"]), "in")
        m = ACTS[block.act](m[:, :block.hidden]) * (m[:, block.hidden:] if block.gated else 1.0)
        y[b][fg[b]] = t + product(m, "down")
    return y


def far(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gated,act,biases", [(True, 1, True), (False, 2, False)])
@pytest.mark.parametrize("in_eight", [False, True])
def test_block_on_slices(dtype, gated, act, biases, in_eight):
    pos = torch.from_numpy(latent_maps(C2.name, 2)).to(DEV)
    block = block_for(pos, dtype, gated, act, biases=biases)
    if in_eight:
        block.lay_out_in_8_bits()
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    for views in ([0], [1, 4], list(range(pos.shape[1]))):
        x = torch.randn((2, len(views)) + tuple(pos.shape[2:4]) + (64,), generator=g, device=DEV).to(dtype)
        before = x.clone()
        got = block(x, views)
        assert torch.equal(x, before) and got.dtype == dtype and got.shape == x.shape
        assert bool((got[~block.foreground[:, views]] == 0).all())
        half = torch.finfo(dtype).eps / 2
        # float32: sums of up to 2^10 terms beside the roundings; 8 bits: borders that go the other way in 0.1 % of the values at most
        bound = 24 * half + (2 ** 10 * half if dtype == torch.float32 else 0)
        if in_eight:
            bound = 2 * bound + 4 * 2.0 ** -4 * math.sqrt(1e-3 if dtype == torch.float32 else 2.0 ** -3)
        assert far(got, plain(block, x, views)) < bound
        assert torch.equal(block(x, views), got)


def test_block_refusals_and_empty_slices():
    pos = torch.from_numpy(latent_maps(C2.name, 1)).to(DEV).clone()
    pos[:, 2] = math.nan
    block = block_for(pos, torch.bfloat16)
    x = torch.randn((1, 1) + tuple(pos.shape[2:4]) + (64,), device=DEV).bfloat16()
    assert bool((block(x, [2]) == 0).all())
    with pytest.raises(ValueError, match="x must be"):
        block(x.float(), [0])
    with pytest.raises(ValueError, match="x must be"):
        block(x, [0, 1])
    with pytest.raises(ValueError, match="views"):
        block(x, [99])
    block.w_down.requires_grad_(True)
    with pytest.raises(ValueError, match="no gradient"):
        block(x, [0])
    with torch.no_grad():
        block(x, [0])
    with pytest.raises(ValueError, match="whole 16"):
        block_for(pos, torch.bfloat16, hidden=168).lay_out_in_8_bits()


def test_block_on_two_streams():
    pos = torch.from_numpy(latent_maps(C2.name, 1)).to(DEV)
    block = block_for(pos, torch.bfloat16)
    block.lay_out_in_8_bits()
    xs = [torch.randn((1, 2) + tuple(pos.shape[2:4]) + (64,), device=DEV).bfloat16() for _ in range(2)]
    want = [block(x, [0, 3]) for x in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for x in xs:
            with torch.cuda.stream(torch.cuda.Stream()):
                got.append(block(x, [0, 3]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_block_in_a_graph():
    """A captured call on a slice that is known, replayed on new inputs between eager calls."""
    pos = torch.from_numpy(latent_maps(C2.name, 1)).to(DEV)
    block = block_for(pos, torch.bfloat16)
    place = torch.randn((1, 2) + tuple(pos.shape[2:4]) + (64,), device=DEV).bfloat16()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block(place, [0, 3])
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = block(place, [0, 3])
    for k in range(4):
        place.copy_(torch.randn(place.shape, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, block(place, [0, 3]))


@pytest.mark.parametrize("in_eight", [False, True])
def test_block_as_denoiser(in_eight):
    """The cached loop's denoiser on the anchors' tokens: a trajectory runs through, twice the same."""
    import paper_2608_13255_amd as gc
    import synth
    from paper_2608_13255_amd.runner import GeoCacheRunner
    w = C4 if C4.N <= 12 else C2
    pos = torch.from_numpy(latent_maps(w.name, 1)).to(DEV)
    cams = gc.camera_tensor({k: v[:1] for k, v in synth.batch_cameras(w).items()}, DEV)
    block = block_for(pos, torch.bfloat16)
    if in_eight:
        block.lay_out_in_8_bits()
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    C = 16
    w_in = (torch.randn((C, 64), generator=g, device=DEV) / 4).bfloat16()
    w_out = (torch.randn((64, C), generator=g, device=DEV) / 8).bfloat16()
    x_T = torch.randn((1, pos.shape[1]) + tuple(pos.shape[2:4]) + (C,), generator=g, device=DEV).bfloat16()
    ends = []
    for _ in range(2):
        runner = GeoCacheRunner(pos, cams, a=2, K=4, sampler=gc.Sampler(kind=gc.GC_FLOW_EULER), S=8,
                                full=GeoCacheRunner.full_steps("head_mid_tail", S=8))
        runner.start(x_T.clone())
        runner.run(lambda k, views: (block(runner.x_t[:, views] @ w_in, views) @ w_out).contiguous())
        ends.append(runner.x_t.clone())
    assert bool(torch.isfinite(ends[0].float()).all()) and torch.equal(ends[0], ends[1])
