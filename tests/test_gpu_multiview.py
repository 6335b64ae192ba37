"""The multi-view attention layer on slices of the views, alone and as the
denoiser of the cached loop, against a plain float64 form of the same layer on
the CPU.

Tolerances: the layer's own bfloat16 roundings (projection, normed and turned
heads, weights, output, each at most 2^-8 of its value) pass through sums of
random signs; their relative effect on the layer's output in the 2-norm is below
sqrt(6) 2^-8 < 1 % when they are independent and below 6 * 2^-8 = 2.4 % in any case.
In float32 the same roundings are 2^-24, and sums of up to 2^13 terms keep the
2-norm within 2^-24 * (2^13 + 100) < 5e-4 in any case.
"""
import math

import pytest
import torch

from synth.configs import C2, C4

from conftest import latent_maps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def layer_for(pos, dtype, width=64, heads=4, kv_heads=2, dim=64):
    from paper_2608_13255_amd.multiview import MultiViewAttention
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    layer = MultiViewAttention(pos, width, heads, kv_heads, dim, dtype, generator=g)
    layer.q_gain.copy_(1 + 0.2 * torch.randn(dim, generator=g, device=DEV))
    layer.k_gain.copy_(1 + 0.2 * torch.randn(dim, generator=g, device=DEV))
    return layer


def plain(layer, x, views, base=10000.0):
    """The layer in float64: asset by asset, head by head."""
    B, n, H, W, _ = x.shape
    h, hk, D = layer.heads, layer.kv_heads, layer.dim
    fg = layer.foreground[:, list(views)].cpu()
    x = x.double().cpu()
    w, wo = layer.w_qkv.double().cpu(), layer.w_out.double().cpu()
    gq, gk = layer.q_gain.double().cpu(), layer.k_gain.double().cpu()
    freq = torch.cat([base ** (-torch.arange(m, dtype=torch.float64) / m) for m in layer.sections])
    axis = torch.cat([torch.full((m,), a) for a, m in enumerate(layer.sections)])
    y = torch.zeros_like(x)
    for b in range(B):
        at = fg[b].nonzero()
        t = x[b][fg[b]] @ w
        q, k, v = t.view(-1, h + 2 * hk, D).split([h, hk, hk], 1)
        place = torch.stack([torch.tensor(list(views))[at[:, 0]], at[:, 1], at[:, 2]], 1).double()
        angle = (place[:, axis] * freq)[:, None]
        c, s = angle.cos(), angle.sin()

        def turn(u, gain):
            u = u / (u.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain
            p, r = u[..., :D // 2], u[..., D // 2:]
            return torch.cat([p * c - r * s, r * c + p * s], -1)

        q, k = turn(q, gq), turn(k, gk)
        o = torch.stack([torch.softmax(q[:, i] @ k[:, i * hk // h].t() / math.sqrt(D), -1) @ v[:, i * hk // h]
                         for i in range(h)], 1)
        y[b][fg[b]] = o.reshape(-1, h * D) @ wo
    return y


def off(got, want):
    d = got.double().cpu() - want
    return float(d.norm() / want.norm())


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 5e-4), (torch.bfloat16, 0.024)], ids=["f32", "bf16"])
@pytest.mark.parametrize("views", [[0], [1, 4], [5, 0, 2], [0, 1, 2, 3, 4, 5]], ids=str)
def test_layer_on_a_slice(views, dtype, tol):
    pos = torch.from_numpy(latent_maps(C2.name)).to(DEV)[:, :, ::2, ::2].contiguous()   # 32 x 32 tokens a view
    layer = layer_for(pos, dtype)
    g = torch.Generator(device=DEV)
    g.manual_seed(len(views))
    x = torch.randn((1, len(views), 32, 32, 64), generator=g, device=DEV).to(dtype)
    y = layer(x, views)
    want = plain(layer, x, views)
    assert off(y, want) < tol
    fg = layer.foreground[:, views]
    assert not y[~fg].any() and bool(y[fg].isfinite().all())
    assert torch.equal(layer(x, views), y)


def test_tokens_keep_their_place_among_all_views():
    """The rotary slots of a slice are those of the full set, and the order of
    the list changes nothing but the order of the result."""
    pos = torch.from_numpy(latent_maps(C2.name)).to(DEV)[:, :, ::4, ::4].contiguous()
    layer = layer_for(pos, torch.float32)
    full = layer.slice(range(6))
    part = layer.slice([4, 1])
    for place, view in enumerate([4, 1]):
        rows = part.positions[(part.index // 256) == place]
        assert torch.equal(rows, full.positions[full.positions[:, 0] == view])
    x = torch.randn((1, 2, 16, 16, 64), device=DEV)
    a, b = layer(x, [4, 1]), layer(x.flip(1), [1, 4])
    assert torch.allclose(a, b.flip(1), rtol=0, atol=1e-4)


@pytest.mark.parametrize("B", [1, 3])
def test_the_cached_loop_with_the_layer_as_its_denoiser(B):
    """Six steps of the runner; each step's prediction against the plain form
    on the state that the step began with."""
    import paper_2608_13255_amd as gc
    import synth
    from paper_2608_13255_amd.runner import GeoCacheRunner
    w = synth.shrink(C4, B=1)
    P = torch.from_numpy(latent_maps(C4.name)).to(DEV)[:, :, ::4, ::4].contiguous()
    P = torch.cat([P, P.roll(1, 1), P.flip(3)])[:B].contiguous()
    cams = gc.camera_tensor({k: v.repeat(B, 0) for k, v in synth.batch_cameras(w).items()}, DEV)
    S, C = 6, 4
    runner = GeoCacheRunner(P, cams, a=3, K=4, sampler=gc.Sampler(kind=gc.GC_FLOW_EULER), S=S,
                            full=GeoCacheRunner.full_steps("periodic", S, 3))
    layer = layer_for(P, torch.bfloat16)
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    w_in = torch.randn((C, 64), generator=g, device=DEV).bfloat16()
    w_back = (torch.randn((64, C), generator=g, device=DEV) / 8).bfloat16()
    asked = []

    def predict(k, views):
        x = runner.x_t[:, views]
        hidden = x @ w_in
        asked.append(list(views))
        y = layer(hidden, views)
        assert off(y, plain(layer, hidden, views)) < 0.024, f"step {k}"
        return (hidden + y) @ w_back

    runner.start(torch.randn((B, 10, 24, 24, C), generator=g, device=DEV).bfloat16())
    runner.run(predict)
    assert [len(v) for v in asked] == [10, 3, 3, 10, 3, 3]
    assert bool(runner.x_t.isfinite().all())
