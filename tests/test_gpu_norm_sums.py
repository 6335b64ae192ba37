"""The sum of squares of a norm where a lane adds the most of them.

With u = 2^-24: bfloat16 rows of 2049 to 4096 columns that are no whole groups lie in one wave, 64 squares a lane.  They are
added one after the other and then in six levels, so the sum is off by at most 69 u of itself, its mean by 71 u with the
reciprocal width and the addition of eps, and the root's reciprocal by 36 u with its own; the products with it and the gain
add 2 u: 38 u of a value.  The scale of a row in 8 bits is off by that and two roundings, 40 u; nothing else rounds it, so it
shows the sum as it is."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


@pytest.mark.parametrize("width", [2049, 2731, 4001, 4095])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows", ["random", "equal", "growing", "one large"])
def test_scale(gc, width, residual, rows):
    g = torch.Generator(device=DEV)
    g.manual_seed(width)
    n = 200
    if rows == "equal":            # roundings of one sign
        x = torch.rand((n, 1), generator=g, device=DEV).expand(n, width) + 0.5
    else:
        x = torch.randn((n, width), generator=g, device=DEV)
        if rows == "growing":
            x *= torch.linspace(0.01, 3, width, device=DEV)
        elif rows == "one large":  # a square that the others hardly change
            x[torch.arange(n), torch.randint(0, width, (n,))] = 3000.0
    x = x.bfloat16().contiguous()
    r = x.flip(1).contiguous() if residual else None
    gain = torch.rand((width,), generator=g, device=DEV) + 0.5
    q, scale, _ = gc.gc_add_rms_norm(x, residual=r, gain=gain, out_dtype=torch.float8_e4m3fn)
    # (the sum as float32 holds it, as the operator does)
    h = x.double() if r is None else (x.float() + r.float()).double()
    want = (h / (h.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain.double()).abs().amax(-1) / 448
    assert float(((scale.double() - want).abs() / want).max()) <= 40 * U
