"""Norms and matrix products of more rows than any one launch takes: the rest go out in launches of their own, with every
pointer moved on.

A launch has at most 2^21 blocks of norms, whose 256 threads or more take at most a row each, and at most 2^20 tiles of a
product, of at most 256 rows.  So 2^29 and 2^28 rows are past a launch of any variant.  Inputs are small whole numbers, so
that sums are exact in every type here, and differ from row to row, so that a row taken for another shows."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NORM_ROWS = (1 << 29) + 1237
LINEAR_ROWS = (1 << 28) + 100003
PIECE = 1 << 24


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def whole(shape, lo, hi, dtype, seed):
    """Whole numbers in [lo, hi], in pieces."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for part in out.split(PIECE):
        part.copy_(torch.randint(lo, hi + 1, part.shape, generator=g, device=DEV, dtype=torch.int8))
    return out


def pieces(n):
    return [slice(i, min(i + PIECE, n)) for i in range(0, n, PIECE)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("where", ["apart", "in place"])
def test_norm(gc, eight, where):
    """One column: h / sqrt(h^2) is the sign of h (off by a few 2^-24, which bfloat16 rounds away)."""
    n = NORM_ROWS
    x, r = whole((n, 1), 1, 3, torch.bfloat16, 1), whole((n, 1), -9, -5, torch.bfloat16, 2)
    r[::2] += 12                                                  # sums of -8 .. -2 and 4 .. 10
    seen = r.clone() if where == "in place" else r
    out, scale, total = gc.gc_add_rms_norm(x, residual=r, gain=torch.full((1,), 2.0, device=DEV), eps=0.0,
                                           out_dtype=torch.float8_e4m3fn if eight else None,
                                           total=r if where == "in place" else None)
    assert (total is r) == (where == "in place")
    for at in pieces(n):
        h = x[at].float() + seen[at].float()
        assert torch.equal(total[at].float(), h)
        assert torch.equal(out[at].float(), torch.sign(h) * (448 if eight else 2))
        if eight:
            assert float((scale[at] * 224 - 1).abs().max()) <= 16 * 2.0 ** -24


def test_quantize(gc):
    n = NORM_ROWS
    x = whole((n, 1), 1, 100, torch.bfloat16, 3)
    x[::3] *= -1
    out, scale = gc.gc_quantize_rows(x)
    for at in pieces(n):
        a = x[at].float()
        assert torch.equal(out[at].float(), torch.sign(a) * 448)
        # (448 times the rounded quotient, rounded)
        assert float((scale[at] * 448 / a[:, 0].abs() - 1).abs().max()) <= 3 * 2.0 ** -24


def test_linear_float32(gc):
    """The output on the residual."""
    n = LINEAR_ROWS
    x, w = whole((n, 4), -4, 4, torch.float32, 4), whole((1, 4), -4, 4, torch.float32, 5)
    r = whole((n, 1), -9, 9, torch.float32, 6)
    seen = r.clone()
    bias = torch.full((1,), 3.0, device=DEV)
    assert gc.gc_linear(x, w, bias=bias, residual=r, out=r) is r
    for at in pieces(n):
        assert torch.equal(r[at], (x[at] * w).sum(1, keepdim=True) + 3 + seen[at])


@pytest.mark.parametrize("gated", [False, True])
def test_linear_in_8_bits(gc, gated):
    """A scale for each row of x: a half, 1 or 2.  Sums of at most 16, so 32 with their scale, in halves."""
    n = LINEAR_ROWS
    x = whole((n, 16), -1, 1, torch.float8_e4m3fn, 7)
    w = torch.ones((1, 16), device=DEV)
    w[0, ::3] = -1
    if gated:                                                     # the value's row: 1 for a scale of 1
        w = torch.cat([w, torch.zeros((1, 16), device=DEV)])
    xs = torch.exp2(whole((n,), -1, 1, torch.float32, 8))
    r = whole((n, 1), -3, 3, torch.bfloat16, 9)
    bias = torch.tensor([0.0, 2.0], device=DEV) if gated else None
    out = gc.gc_linear(x, w.to(torch.float8_e4m3fn), bias=bias, gated=gated, x_scale=xs,
                       w_scale=torch.ones(w.shape[0], device=DEV), residual=r)
    assert out.dtype == torch.bfloat16
    for at in pieces(n):
        p = (x[at].float() * w[:1]).sum(1, keepdim=True) * xs[at][:, None]
        assert torch.equal(out[at].float(), p * (2 if gated else 1) + r[at].float())
