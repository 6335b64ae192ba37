"""gc_linear where the products cancel: every sum is 0 by the formula, so what comes out is the sum's own error, relative to the
products.

Float32 sums are off by at most K u of the magnitudes' sum, u = 2^-24, in any order.  The 8-bit units cut each of 64 terms at
2^-13 of the largest at worst: 2^-7 of each 64 columns' largest product, added up."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "f32"), ("e4m3", "f32"), ("e4m3", "bf16")])
@pytest.mark.parametrize("M", [3, 16, 17, 200])
@pytest.mark.parametrize("K", [64, 512, 4096])
@pytest.mark.parametrize("large", [False, True])
def test_sums_that_cancel(kind, out, M, K, large):
    import paper_2608_13255_amd as gc
    g = torch.Generator(device=DEV)
    g.manual_seed(M + K)
    N, half = 130, K // 2
    a, b = torch.randn((M, half), generator=g, device=DEV), torch.randn((N, half), generator=g, device=DEV)
    if large:                                   # one channel in 64
        a[:, torch.randperm(half, generator=g, device=DEV)[:max(1, half // 64)]] *= 100
    a, b = ((t / t.abs().amax(-1, keepdim=True) * 448).to(TYPES[kind]).float() for t in (a, b))
    order = torch.randperm(K, generator=g, device=DEV)
    x, w = (torch.cat(t, 1)[:, order].to(TYPES[kind]) for t in ((a, a), (b, -b)))
    got = gc.gc_linear(x, w, out_dtype=TYPES[out]).double()
    x, w = x.double(), w.double()
    if kind == "e4m3" and out == "bf16" and M > 16:
        bound = sum((x[:, None, k:k + 64] * w[None, :, k:k + 64]).abs().amax(-1) for k in range(0, K, 64)) * 2.0 ** -7
    else:
        bound = K * U * (x.abs() @ w.abs().t())
    # (the store rounds what is there by half a step)
    assert float((got.abs() - bound * (1 + torch.finfo(TYPES[out]).eps / 2)).max()) <= 0
