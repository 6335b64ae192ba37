"""gc_add_rms_norm and gc_quantize_rows against the same in 64 bits.

Bounds, with u = 2^-24: a row's squares are added by lanes of at most 32 values
and a tree, so their mean is off by at most 40 u of itself and its root by half of
that; the products with it and the gain, and h's own rounding, add a few u.  A scale is off by as much and one
more.  The stored value is rounded by half a step: of its type, or of e4m3, 2^-4 of the
quotient and 2^-10 where that is subnormal."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
WIDTHS = [1, 2, 7, 8, 16, 63, 64, 72, 512, 520, 1000, 1024, 1283, 2048, 2056, 4096, 4104, 8192, 8200, 16384, 20000, 32768]


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


def rows(n, width, dtype, seed, pad=0, size=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn((n, width + pad), generator=g, device=DEV) * size).to(dtype)[:, pad // 2:pad // 2 + width]


def norm64(x, r, gain, eps):
    h = x.double() + (0 if r is None else r.double())
    y = h / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    return h, y if gain is None else y * gain.double()


def near(got, want, rel, extra=0.0):
    step = torch.finfo(got.dtype).eps / 2
    bad = (got.double() - want).abs() - (rel + step) * 1.001 * want.abs() - extra - torch.finfo(got.dtype).tiny
    assert float(bad.max()) <= 0, (float((got.double() - want).abs().max()), float(bad.max()))


def near_eight(q, scale, want, rel):
    """8-bit rows and their scales against rows in 64 bits."""
    top = want.abs().amax(-1).clamp_min(448 * 2.0 ** -126) / 448
    assert float(((scale.double() - top).abs() - (rel + 2 * U) * top).max()) <= 0
    value, s = q.double(), scale.double()[:, None]
    bad = (value * s - want).abs() - (rel + 2.0 ** -4 * (1 + rel) + 4 * U) * want.abs() - s * 2.0 ** -10
    assert float(bad.max()) <= 0


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("eight", [False, True])
def test_norm(gc, width, dtype, residual, eight):
    n = 37 if width < 5000 else 5
    x = rows(n, width, dtype, 1)
    r = rows(n, width, dtype, 2, size=3.0) if residual else None
    gain = rows(1, width, torch.float32, 3)[0]
    out, scale, total = gc.gc_add_rms_norm(x, residual=r, gain=gain, eps=1e-5, out_dtype=torch.float8_e4m3fn if eight else None)
    h, y = norm64(x, r, gain, 1e-5)
    # (h is rounded once: u of h, and through the norm at most 2 u of the result and u of the row's scale of h)
    h_off = U * (x.double().abs() + (0 if r is None else r.double().abs()))
    extra = (h_off / h.abs().clamp_min(1e-300) * y.abs()) if residual else torch.zeros_like(y)
    if residual:
        near(total, h, U)
    else:
        assert total is x
    if eight:
        assert out.dtype == torch.float8_e4m3fn
        near_eight(out, scale, y, 60 * U)
    else:
        assert scale is None
        near(out, y, 30 * U, extra)


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize(gc, width, dtype):
    x = rows(37 if width < 5000 else 5, width, dtype, 4, size=20.0)
    q, scale = gc.gc_quantize_rows(x)
    near_eight(q, scale, x.double(), 0.0)
    # the quotient is rounded to the nearest: exactly what a division in 64 bits rounds to, off ties within float32's error
    want = (x.double() / scale.double()[:, None])
    nearest = want.float().to(torch.float8_e4m3fn)
    assert float((q.float() != nearest.float()).float().mean()) <= 1e-4


@pytest.mark.parametrize("n", [1, 3, 4, 5, 255, 4097])
@pytest.mark.parametrize("width", [40, 1001])
def test_row_counts(gc, n, width):
    x = rows(n, width, torch.bfloat16, 5)
    guard = torch.full((n + 2, width), 9.0, dtype=torch.bfloat16, device=DEV)
    out, _, _ = gc.gc_add_rms_norm(x, out=guard[1:-1])
    near(out, norm64(x, None, None, 1e-6)[1], 30 * U)
    assert bool((guard[0] == 9).all()) and bool((guard[-1] == 9).all())


def test_no_rows(gc):
    x = torch.empty((0, 64), device=DEV)
    out, scale, total = gc.gc_add_rms_norm(x, residual=x, out_dtype=torch.float8_e4m3fn)
    assert out.shape == (0, 64) and scale.shape == (0,) and total.shape == (0, 64)
    assert gc.gc_quantize_rows(x)[0].shape == (0, 64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width,pad", [(64, 16), (100, 7), (2048, 32), (1283, 2), (4000, 3), (9001, 5), (20000, 6), (32768, 2)])
def test_strides(gc, dtype, width, pad):
    """Columns of wider buffers, aligned and not; what lies around the outputs stays."""
    x, r = rows(50, width, dtype, 6, pad), rows(50, width, dtype, 7, pad)
    buffer = torch.full((50, width + pad), 5.0, dtype=dtype, device=DEV)
    total = buffer[:, pad // 2:pad // 2 + width]
    eight = torch.full((50, width + pad), 3.0, device=DEV).to(torch.float8_e4m3fn)
    for out in (None, eight[:, pad // 2:pad // 2 + width]):
        got, scale, t = gc.gc_add_rms_norm(x, residual=r, total=total, out=out)
        assert t is total
        h, y = norm64(x, r, None, 1e-6)
        near(total, h, U)
        if out is None:
            extra = U * (x.double().abs() + r.double().abs()) / h.abs().clamp_min(1e-300) * y.abs()
            near(got, y, 30 * U, extra)
        else:
            near_eight(got, scale, y, 60 * U)
    total.fill_(5.0)
    assert bool((buffer == 5).all())
    eight[:, pad // 2:pad // 2 + width] = torch.full((50, width), 3.0, device=DEV).to(torch.float8_e4m3fn)
    assert bool((eight.float() == 3).all())


def test_in_place(gc):
    for width in (1000, 4096):
        x, r = rows(20, width, torch.bfloat16, 8), rows(20, width, torch.bfloat16, 9)
        want, _, want_total = gc.gc_add_rms_norm(x, residual=r)
        for total_on, out_on in (("x", None), ("r", None), ("x", "r"), ("r", "x"), (None, "x")):
            place = {"x": x.clone(), "r": r.clone()}
            out, _, total = gc.gc_add_rms_norm(place["x"], residual=place["r"], total=place.get(total_on), out=place.get(out_on))
            assert torch.equal(out, want) and torch.equal(total, want_total)
            assert (total_on is None or total is place[total_on]) and (out_on is None or out is place[out_on])


def test_a_residual_of_one_row(gc):
    x, r = rows(9, 256, torch.float32, 10), rows(1, 256, torch.float32, 11)
    a = gc.gc_add_rms_norm(x, residual=r.expand(9, -1))
    b = gc.gc_add_rms_norm(x, residual=r.expand(9, -1).contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


@pytest.mark.parametrize("width", [24, 100, 3000])
def test_rows_of_zeros_and_nonfinite(gc, width):
    """A row of zeros has scale 2^-126 and zeros (with eps 0 its norm is 0 / 0); a NaN or infinity marks its own row alone."""
    for dtype in (torch.float32, torch.bfloat16):
        x = rows(6, width, dtype, 12)
        x[1] = 0
        x[2, width - 1] = math.nan
        x[3, 0] = -math.inf
        q, scale = gc.gc_quantize_rows(x)
        assert float(scale[1]) == 2.0 ** -126 and bool((q[1].float() == 0).all())
        assert bool(torch.isnan(scale[2:4]).all()) and bool(torch.isnan(q[2:4].float()).all())
        near_eight(q[4:], scale[4:], x[4:].double(), 0.0)
        out, _, _ = gc.gc_add_rms_norm(x)
        assert bool((out[1] == 0).all()) and bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3, 0]))
        near(out[4:], norm64(x[4:], None, None, 1e-6)[1], 30 * U)
        out, scale, _ = gc.gc_add_rms_norm(x, eps=0.0, out_dtype=torch.float8_e4m3fn)
        assert bool(torch.isnan(scale[1:4]).all()) and bool(torch.isnan(out[1:4].float()).all())


def test_small_and_large_values(gc):
    """Down to float32's subnormals the quotient is right to its step; the largest values are taken too."""
    for size in (1e-38, 1e-30, 1e30, 1e37):
        x = (rows(4, 512, torch.float32, 13).clamp(-8, 8) * size)
        q, scale = gc.gc_quantize_rows(x)
        assert bool(torch.isfinite(scale).all())
        value, s = q.double(), scale.double()[:, None]
        # (below the smallest scale the quotient's float32 arithmetic is exact to 2^-149)
        bad = (value * s - x.double()).abs() - (2.0 ** -4 + 4 * U) * x.double().abs() - s * 2.0 ** -10 - 2.0 ** -148
        assert float(bad.max()) <= 0
    for size in (1e-15, 1e15):
        x = rows(4, 512, torch.float32, 14) * size
        near(gc.gc_add_rms_norm(x, eps=0.0)[0], norm64(x, None, None, 0.0)[1], 30 * U)


def test_offsets_past_32_bits(gc):
    n, width, far = 70, 128, 2 ** 26
    x = rows(n, width, torch.bfloat16, 15)
    place = torch.empty((n - 1) * far + width, dtype=torch.bfloat16, device=DEV).as_strided((n, width), (far, 1))
    place.copy_(x)
    want, _, _ = gc.gc_add_rms_norm(x)
    assert torch.equal(gc.gc_add_rms_norm(place)[0], want)
    assert torch.equal(gc.gc_add_rms_norm(place, out=place)[0], want)


def test_more_rows_than_a_launch_has(gc):
    """Rows past one launch's blocks go out in the next one."""
    n = (1 << 23) + 5
    x = torch.randint(-3, 4, (n, 1), device=DEV, dtype=torch.int8).to(torch.bfloat16)
    q, scale = gc.gc_quantize_rows(x)
    some = x.float() != 0
    assert bool((q.float()[some].abs() == 448).all()) and bool((q.float()[~some] == 0).all())
    assert bool(((scale * 448)[:, None][some] == x.float().abs()[some]).all())


def test_graph_replays_and_streams(gc):
    x, r = rows(300, 1283, torch.float32, 16), rows(300, 1283, torch.float32, 17)
    place = x.clone()
    call = lambda: gc.gc_add_rms_norm(place, residual=r, out_dtype=torch.float8_e4m3fn)
    want = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for k in range(4):
        place.copy_(x * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        again = call()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, again))
    s = torch.cuda.Stream()
    place.copy_(x)
    torch.cuda.synchronize()
    side = gc.gc_add_rms_norm(place, residual=r, out_dtype=torch.float8_e4m3fn, stream=s)
    s.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(side, want))


def test_refusals_on_the_device(gc):
    x = torch.zeros((4, 32), device=DEV)
    with pytest.raises(ValueError, match="residual"):
        gc.gc_add_rms_norm(x, residual=x[:, :16])
    with pytest.raises(ValueError, match="gain"):
        gc.gc_add_rms_norm(x, gain=torch.ones(16, device=DEV))
    with pytest.raises(ValueError, match="rows must be"):
        gc.gc_add_rms_norm(x.half())
    with pytest.raises(gc.GeoCacheError, match="out_dtype"):
        gc.gc_add_rms_norm(x, out_dtype=torch.bfloat16)
    with pytest.raises(gc.GeoCacheError, match="width"):
        gc.gc_add_rms_norm(torch.zeros((2, 40000), device=DEV))
    with pytest.raises(gc.GeoCacheError, match="out overlaps x"):
        y = torch.zeros((4, 48), device=DEV)
        gc.gc_add_rms_norm(y[:, :32], out=y[:, 8:40])
    with pytest.raises(gc.GeoCacheError, match="rows overlap"):
        gc.gc_add_rms_norm(x, out=torch.zeros((1, 32), device=DEV).expand(4, -1))
    with pytest.raises(gc.GeoCacheError, match="out_scale"):
        gc.gc_add_rms_norm(x, out_scale=torch.zeros(4, device=DEV))


def test_sizes_past_32_bits_are_refused(gc):
    x = torch.ones((1, 16), device=DEV)
    for call in (gc.gc_add_rms_norm, gc.gc_quantize_rows):
        with pytest.raises(ValueError, match="2\\^31"):
            call(x.expand(2 ** 32 + 3, 16))
    with pytest.raises(ValueError, match="2\\^31"):
        gc.gc_linear(x, x.expand(2 ** 32 + 3, 16))


# odd widths, whose last 16 bytes overlap the ones before: in parts of a wave, one wave, and several that store while others read
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", [9, 67, 131, 517, 1283, 4099, 9001, 20001, 32767])
def test_odd_rows_in_place(gc, dtype, width):
    n = 300
    x, r = rows(n, width, dtype, 30), rows(n, width, dtype, 31)
    gain = rows(1, width, torch.float32, 32)[0]
    want, _, total = gc.gc_add_rms_norm(x, residual=r, gain=gain)
    assert torch.equal(total, (x.float() + r.float()).to(dtype))
    for times in range(3):
        a, b = x.clone(), r.clone()
        gc.gc_add_rms_norm(a, residual=b, gain=gain, total=a, out=b)
        assert torch.equal(a, total) and torch.equal(b, want)
        a, b = x.clone(), r.clone()
        gc.gc_add_rms_norm(a, residual=b, gain=gain, total=b, out=a)
        assert torch.equal(b, total) and torch.equal(a, want)
    eight, scale, _ = gc.gc_add_rms_norm(x, residual=r, gain=gain, out_dtype=torch.float8_e4m3fn)
    a = x.clone()
    got, got_scale, _ = gc.gc_add_rms_norm(a, residual=r, gain=gain, total=a, out_dtype=torch.float8_e4m3fn)
    assert torch.equal(a, total) and torch.equal(got.view(torch.uint8), eight.view(torch.uint8)) and torch.equal(got_scale, scale)
