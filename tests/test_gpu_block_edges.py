"""Slices on which a block has little or nothing to do, in its own type and in 8 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def block_for(dtype, eight, foreground):
    """A block on two assets of three 4 x 5 views; foreground: (asset, view, row, column) of its tokens."""
    from paper_2608_13255_amd.multiview import MultiViewBlock
    g = torch.Generator(device=DEV)
    g.manual_seed(40)
    pos = torch.full((2, 3, 4, 5, 3), math.nan, device=DEV)
    for at in foreground:
        pos[at] = 0.5
    block = MultiViewBlock(pos, 32, 2, 1, 16, 48, dtype=dtype, generator=g)
    if eight:
        block.lay_out_in_8_bits()
    return block, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("views", [[], [1], [1, 2]])
def test_nothing_in_the_foreground(dtype, eight, views):
    block, g = block_for(dtype, eight, [(0, 0, 1, 1)])
    x = torch.randn((2, len(views), 4, 5, 32), generator=g, device=DEV).to(dtype)
    y = block(x, views)
    assert y.shape == x.shape and y.dtype == dtype and bool((y == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("eight", [False, True])
def test_a_token_alone(dtype, eight):
    """One token attends to itself alone: the same result wherever it lies and whatever the background holds.  Not bit for bit:
    its score depends on its place (the rotation is rounded), and its weight, e^(s - s) by float32's products, is 1 up to a
    rounding before it is divided by itself.  A block's result is off by less than 24 half steps of its type, and by 2^10 of them
    for float32's sums, in the 2-norm (twelve roundings, gains and norms keep that norm within a factor of two): two results
    differ by twice that at most."""
    block, g = block_for(dtype, eight, [(0, 0, 1, 1), (1, 2, 3, 4)])
    t = torch.randn((32,), generator=g, device=DEV).to(dtype)
    results = []
    for asset, view, row, col in ((0, 0, 1, 1), (1, 2, 3, 4)):
        x = torch.full((2, 1, 4, 5, 32), math.nan, dtype=dtype, device=DEV)
        x[asset, 0, row, col] = t
        y = block(x, [view])
        assert bool(torch.isfinite(y).all())
        results.append(y[asset, 0, row, col].clone())
        y[asset, 0, row, col] = 0
        assert bool((y == 0).all())
    a, b = (r.double() for r in results)
    assert bool(a.any()) and bool(b.any())
    if not eight:      # (8-bit rows may round a border the other way)
        half = torch.finfo(dtype).eps / 2
        assert float((a - b).norm() / a.norm()) <= 2 * (24 + (2 ** 10 if dtype == torch.float32 else 0)) * half
