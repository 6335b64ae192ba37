"""gc_linear against products in 64 bits: every operand type, variant (few rows,
tiles of every size, parts of the inner dimension), epilogue and edge.

Bounds: a float32 sum of K products in any order is off by at most K u S with
u = 2^-24 and S the sum of the products' magnitudes; the epilogue's operations
and functions add a few u of their results, and activations have slopes of at
most 1.13.  8-bit products with a bfloat16 result cut each of 64 terms at 2^-13 of
the largest at worst: off by 2^-7 of each 64 columns' largest product.  The
stored value is rounded by half a step."""
import itertools
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
ACTS = ["none", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


def act64(p, act):
    if act == "silu":
        return p * torch.sigmoid(p)
    if act == "gelu":
        return p * torch.special.erfc(-p / math.sqrt(2)) / 2
    if act == "gelu_tanh":
        return p * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (p + 0.044715 * p ** 3))
    return p


def operands(kind, M, R, K, g, wide=0, size=1.0):
    """x (columns of a wider buffer where wide), w, their scales and both in 64 bits."""
    x = torch.randn((M, K + wide), generator=g, device=DEV)
    w = torch.randn((R, K), generator=g, device=DEV) * size / math.sqrt(K)
    if kind != "e4m3":
        x, w = x.to(TYPES[kind])[:, wide // 2:wide // 2 + K], w.to(TYPES[kind])
        return x, w, None, None, x.double(), w.double()
    xs = torch.rand((M,), generator=g, device=DEV) * 0.02 + 0.001
    ws = torch.rand((R,), generator=g, device=DEV) * 0.01 + 0.001
    x8 = torch.empty((M, K + wide), dtype=TYPES[kind], device=DEV)
    x8.copy_((x * 60).clamp(-448, 448))
    x8 = x8[:, wide // 2:wide // 2 + K]
    w8 = (w * math.sqrt(K) * 100).clamp(-448, 448).to(TYPES[kind])
    return x8, w8, xs, ws, x8.double() * xs.double()[:, None], w8.double() * ws.double()[:, None]


def expected(x, w, bias, act, gated, residual, coarse):
    """(result in 64 bits, how far float32 arithmetic may be off before the store)."""
    K = x.shape[1]
    p, s = x @ w.t(), x.abs() @ w.abs().t()
    off = (K + 4) * U * s
    if coarse:
        for k in range(0, K, 64):
            top = (x[:, None, k:k + 64].abs() * w[None, :, k:k + 64].abs()).amax(-1)
            off = off + 2.0 ** -7 * top
    if bias is not None:
        p = p + bias.double()
        off = off + U * p.abs()
    n = p.shape[1] // 2 if gated else p.shape[1]
    y = act64(p[:, :n], act)
    # (the functions themselves: their argument's rounding, 3 u |p|, times at most |p| times the slope of their exponential)
    err = 1.13 * off[:, :n] + (0 if act == "none" else 16 * U * p[:, :n].abs().clamp_min(1.0))
    if gated:
        v = p[:, n:]
        err = err * (v.abs() + off[:, n:]) + off[:, n:] * y.abs() + U * (y * v).abs()
        y = y * v
    if residual is not None:
        y = y + residual.double()
        err = err + U * y.abs()
    return y, err


def check(got, y, err, label=""):
    step = torch.finfo(got.dtype).eps / 2
    bound = err + step * (y.abs() + err) + torch.finfo(got.dtype).tiny
    bad = (got.double() - y).abs() - bound
    assert torch.isfinite(got).all(), label
    assert float(bad.max()) <= 0, (label, float((got.double() - y).abs().max()), float(bad.max()))


def run(gc, kind, out_kind, M, N, K, act="none", gated=False, bias=False, residual=False, wide=0, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 1)
    R = 2 * N if gated else N
    x, w, xs, ws, x64, w64 = operands(kind, M, R, K, g, wide)
    b = torch.randn((R,), generator=g, device=DEV) if bias else None
    r = torch.randn((M, N), generator=g, device=DEV).to(TYPES[out_kind]) if residual else None
    out = gc.gc_linear(x, w, bias=b, act=ACTS.index(act), gated=gated, residual=r, x_scale=xs, w_scale=ws,
                       out_dtype=TYPES[out_kind])
    assert out.shape == (M, N) and out.dtype == TYPES[out_kind]
    check(out, *expected(x64, w64, b, act, gated, r, kind == "e4m3" and out_kind == "bf16"), f"{kind} {M} {N} {K}")
    return out


PAIRS = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("e4m3", "bf16"), ("e4m3", "f32")]


@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 64, 65, 130])
@pytest.mark.parametrize("N,K", [(1, 16), (8, 48), (15, 64), (16, 528), (33, 144), (128, 1024), (200, 2064)])
def test_sizes(gc, kind, out, M, N, K):
    run(gc, kind, out, M, N, K, bias=True)


@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("M,N,K", [(7, 40, 320), (97, 72, 208)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, True)])
def test_epilogues(gc, kind, out, M, N, K, act, gated, bias, residual):
    run(gc, kind, out, M, N, K, act, gated, bias, residual)


# more than eight rows and many weight rows: 32 of them a block, the last block's second 16 whole, one, or none
@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("M,N,K", [(9, 8177, 272), (16, 8193, 1040), (12, 8208, 16), (16, 8224, 4096)])
def test_rows_with_many_weight_rows(gc, kind, out, M, N, K):
    run(gc, kind, out, M, N, K, "gelu", False, True, True)


# every variant, by what the rule on sizes takes there: tiles of 64 (and 32 x 64) and 128, one and two on a compute unit, 192, 256;
# one part, a few and sixteen
@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("M,N,K", [(300, 520, 96), (513, 1000, 1040), (1030, 2050, 304), (1100, 4100, 112), (2300, 1030, 400),
                                   (2900, 4000, 2048), (4000, 4090, 1024), (130, 136, 6000 // 16 * 16), (20, 24, 16384),
                                   (70, 2000, 4096)])
@pytest.mark.parametrize("gated", [False, True])
def test_variants(gc, kind, out, M, N, K, gated):
    g = torch.Generator(device=DEV)
    g.manual_seed(M)
    N = N // 2 if gated else N
    R = 2 * N if gated else N
    x, w, xs, ws, x64, w64 = operands(kind, M, R, K, g)
    b = torch.randn((R,), generator=g, device=DEV)
    r = torch.randn((M, N), generator=g, device=DEV).to(TYPES[out])
    got = gc.gc_linear(x, w, bias=b, act=1, gated=gated, residual=r, x_scale=xs, w_scale=ws, out_dtype=TYPES[out])
    # all of it roughly (a wrong, missing or doubled step or part shows in whole rows or columns), some of it exactly
    p = x64 @ w64.t() + b.double()
    y = act64(p[:, :N], "silu") * (p[:, N:] if gated else 1.0) + r.double()
    assert torch.isfinite(got).all()
    scale = p.std() * (1 + p.std() if gated else 1) + 1
    assert float((got.double() - y).abs().max() / scale) < 0.25
    rows = torch.cat([torch.arange(min(M, 20)), torch.arange(max(0, M - 20), M), torch.randint(0, M, (24,))]).to(DEV)
    cols = torch.cat([torch.arange(min(N, 12)), torch.arange(max(0, N - 12), N), torch.randint(0, N, (8,))]).to(DEV)
    at = torch.cat([cols, N + cols]) if gated else cols
    want, err = expected(x64[rows], w64[at], b[at], "silu", gated, r[rows][:, cols], kind == "e4m3" and out == "bf16")
    check(got[rows][:, cols], want, err)


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "bf16")])
@pytest.mark.parametrize("M,N", [(3, 40), (100, 130), (1500, 2000)])
def test_strides_and_margins(gc, kind, out, M, N):
    """x and w as columns of wider buffers, the output as columns of another: what lies around it stays as it was, what lies
    around the operands, NaN, has no effect."""
    K, pad = 208, 16
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x, w, xs, ws, x64, w64 = operands(kind, M, N, K, g)
    if kind == "e4m3":
        hole = lambda n: torch.full((n, K + 2 * pad), 0x7f, dtype=torch.uint8, device=DEV).view(TYPES[kind])
    else:
        hole = lambda n: torch.full((n, K + 2 * pad), math.nan, dtype=TYPES[kind], device=DEV)
    bx, bw = hole(M + 2), hole(N + 2)
    bx[1:-1, pad:-pad] = x
    bw[1:-1, pad:-pad] = w
    o = torch.full((M + 2, N + 23), 7.0, dtype=TYPES[out], device=DEV)     # rows that are no whole number of 16 bytes
    r = torch.randn((M, N), generator=g, device=DEV).to(TYPES[out])
    for first in (8, 3):
        o.fill_(7.0)
        view = o[1:-1, first:first + N]
        got = gc.gc_linear(bx[1:-1, pad:-pad], bw[1:-1, pad:-pad], residual=r, x_scale=xs, w_scale=ws, out=view)
        assert got is view
        check(view, *expected(x64, w64, None, "none", False, r, kind == "e4m3"))
        view.fill_(7.0)
        assert bool((o == 7.0).all())


@pytest.mark.parametrize("M,N,K", [(5, 64, 128), (90, 128, 4096), (700, 512, 256)])
def test_output_on_the_residual(gc, M, N, K):
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    x, w, _, _, x64, w64 = operands("bf16", M, N, K, g)
    r = torch.randn((M, N), generator=g, device=DEV).bfloat16()
    want, err = expected(x64, w64, None, "gelu", False, r, False)
    got = gc.gc_linear(x, w, act=2, residual=r, out=r)
    assert got is r
    check(r, want, err)


def test_rows_that_repeat(gc):
    """An input's rows may share memory: one row for all, and a residual of one row."""
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    x, w, _, _, x64, w64 = operands("bf16", 1, 96, 320, g)
    r = torch.randn((1, 96), generator=g, device=DEV).bfloat16()
    for M in (9, 200):
        got = gc.gc_linear(x.expand(M, -1), w, residual=r.expand(M, -1))
        check(got, *expected(x64.expand(M, -1), w64, None, "none", False, r.expand(M, -1), False))
        assert bool((got == got[:1]).all())


def test_no_rows(gc):
    w = torch.randn((24, 32), device=DEV)
    assert gc.gc_linear(torch.empty((0, 32), device=DEV), w).shape == (0, 24)


@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("M", [12, 300])
def test_nonfinite_rows_stay_apart(gc, kind, out, M):
    """A NaN or infinity in a row of x reaches that row of the result, one in a weight row its column; no other."""
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    N, K = 100, 176
    x, w, xs, ws, x64, w64 = operands(kind, M, N, K, g)
    clean = gc.gc_linear(x, w, x_scale=xs, w_scale=ws, out_dtype=TYPES[out])
    bad = math.nan if kind == "e4m3" else math.inf
    x, w = x.clone(), w.clone()
    if kind == "e4m3":
        x.view(torch.uint8)[5, K - 1], w.view(torch.uint8)[17, 0] = 0x7f, 0x7f
    else:
        x[5, K - 1], w[17, 0] = bad, -bad
    got = gc.gc_linear(x, w, x_scale=xs, w_scale=ws, out_dtype=TYPES[out])
    assert not torch.isfinite(got[5]).any() and not torch.isfinite(got[:, 17]).any()
    keep = torch.ones((M, N), dtype=torch.bool, device=DEV)
    keep[5], keep[:, 17] = False, False
    assert bool((got[keep] == clean[keep]).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [1, 40])
def test_activations_over_their_range(gc, act, M):
    """One product of 1 a value: the activation of each float itself, far and near, and its limits."""
    p = torch.cat([torch.linspace(-30, 30, 4001), torch.logspace(-30, 18, 97), -torch.logspace(-30, 18, 97),
                   torch.tensor([0.0, 1e19, -1e19, 3e38, -3e38, math.inf])]).to(DEV)
    w = torch.zeros((p.numel(), 4), device=DEV)
    w[:, 0] = p
    x = torch.zeros((M, 4), device=DEV)
    x[:, 0] = 1.0
    got = gc.gc_linear(x, w, act=ACTS.index(act))
    # (0 times an infinite weight is a NaN, so that one is left to the bias)
    got[:, -1] = gc.gc_linear(x, torch.zeros((1, 4), device=DEV), bias=p[-1:].clone(), act=ACTS.index(act))[:, 0]
    want = act64(p.double(), act)
    fine = torch.isfinite(want) & (want.abs() <= 3.4e38)
    # relative 2^-20 of p's own part where the function is not tiny, 2^-22 of |p| at most elsewhere
    bound = 2.0 ** -21 * want.abs() + 2.0 ** -22 * p.double().abs().clamp_max(8.0) + 1e-37
    assert float(((got.double() - want).abs() - bound)[:, fine].max()) <= 0
    assert bool((got[:, -1] == math.inf).all())


@pytest.mark.parametrize("M,N,K", [(2100, 24, 64), (12, 24, 64)])
def test_offsets_past_32_bits(gc, M, N, K):
    """Rows 2^20 elements apart: over 4 GiB of them (12 rows: the output's)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    x, w, _, _, x64, w64 = operands("bf16", M, N, K, g)
    if M > 1000:
        far = torch.empty((M - 1) * 2 ** 20 + K, dtype=torch.bfloat16, device=DEV).as_strided((M, K), (2 ** 20, 1))
        far.copy_(x)
        got = gc.gc_linear(far, w)
    else:
        out = torch.empty(((M - 1) * 2 ** 28 + N,), dtype=torch.bfloat16, device=DEV).as_strided((M, N), (2 ** 28, 1))
        got = gc.gc_linear(x, w, out=out)
    check(got.contiguous(), *expected(x64, w64, None, "none", False, None, False))


def test_more_outputs_than_an_int_counts(gc):
    g = torch.Generator(device=DEV)
    g.manual_seed(9)
    M, N, K = 70000, 32768, 8
    x, w, _, _, x64, w64 = operands("bf16", M, N, K, g)
    got = gc.gc_linear(x, w)
    for i in (0, 33333, M - 1):
        check(got[i:i + 1], *expected(x64[i:i + 1], w64, None, "none", False, None, False))
    assert bool((got[:, 5] == gc.gc_linear(x, w[5:6].clone())[:, 0]).all())
    del got
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind,M,N,K", [("bf16", 9, 64, 256), ("bf16", 200, 136, 8192), ("f32", 513, 300, 512),
                                        ("e4m3", 2000, 2048, 512)])
def test_same_again_and_in_a_graph(gc, kind, M, N, K):
    """Bit for bit the same from call to call, and from a graph's replays with other work between them and new inputs in
    the same place."""
    g = torch.Generator(device=DEV)
    g.manual_seed(10)
    x, w, xs, ws, _, _ = operands(kind, M, N, K, g)
    other = operands(kind, M, N, K, g)[0]
    call = lambda a: gc.gc_linear(a, w, act=1, x_scale=xs, w_scale=ws)
    want, want_other = call(x), call(other)
    for _ in range(3):
        assert torch.equal(call(x), want)
    place = x.clone()
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(place)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        got = call(place)
    for source, result in itertools.chain([(x, want), (other, want_other)] * 3):
        place.copy_(source)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, result)
        call(other).sum().item()          # eager work of the same kind between replays


def test_two_streams_at_once(gc):
    """Calls with parts of the inner dimension on two streams, each with a workspace of its own from the allocator."""
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    jobs = [operands("bf16", 120, 256, 8192, g)[:2] for _ in range(2)]
    assert gc.gc_linear_workspace_bytes(120, 256, 8192, torch.bfloat16) > 0
    want = [gc.gc_linear(*j) for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for s, j in zip(streams, jobs):
            got.append(gc.gc_linear(*j, stream=s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_workspace_of_the_caller(gc):
    g = torch.Generator(device=DEV)
    g.manual_seed(12)
    x, w = operands("bf16", 120, 256, 8192, g)[:2]
    need = gc.gc_linear_workspace_bytes(120, 256, 8192, torch.bfloat16)
    want = gc.gc_linear(x, w)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device=DEV)      # NaN: its contents are of no consequence
    assert torch.equal(gc.gc_linear(x, w, workspace=ws), want)
    assert bool((ws[need:] == 0xff).all())
    with pytest.raises(gc.GeoCacheError, match="workspace"):
        gc.gc_linear(x, w, workspace=ws[:need - 16])


def test_refusals_on_the_device(gc):
    x, w = torch.zeros((4, 32), device=DEV), torch.zeros((6, 32), device=DEV)
    with pytest.raises(ValueError, match="w must be"):
        gc.gc_linear(x, w.bfloat16())
    with pytest.raises(ValueError, match="w must be"):
        gc.gc_linear(x, w[:, :16])
    with pytest.raises(ValueError, match="even number"):
        gc.gc_linear(x, w[:5], gated=True)
    with pytest.raises(ValueError, match="residual"):
        gc.gc_linear(x, w, residual=torch.zeros((4, 5), device=DEV))
    with pytest.raises(ValueError, match="bias"):
        gc.gc_linear(x, w, bias=torch.zeros(5, device=DEV))
    with pytest.raises(ValueError, match="contiguous columns"):
        gc.gc_linear(torch.zeros((32, 4), device=DEV).t(), w)
    with pytest.raises(ValueError, match="columns"):
        gc.gc_linear(x[None], w)
    with pytest.raises(gc.GeoCacheError, match="out_dtype"):
        gc.gc_linear(x, w, out_dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="out_dtype"):
        gc.gc_linear(x, w, out_dtype=torch.float16)
    with pytest.raises(gc.GeoCacheError, match="scales"):
        gc.gc_linear(x, w, x_scale=torch.ones(4, device=DEV))
    with pytest.raises(gc.GeoCacheError, match="n_in"):
        gc.gc_linear(x[:, :30].contiguous(), w[:, :30].contiguous())
    with pytest.raises(gc.GeoCacheError, match="16-byte"):
        gc.gc_linear(torch.zeros((4, 36), device=DEV)[:, 2:34], w)
    with pytest.raises(gc.GeoCacheError, match="activation"):
        gc.gc_linear(x, w, act=9)
    with pytest.raises(gc.GeoCacheError, match="overlaps x"):
        gc.gc_linear(x, w, out=x[:, :6])


@pytest.mark.parametrize("M", [7, 150])
def test_x_and_output_in_one_buffer(gc, M):
    """The output beside x in the rows of one buffer."""
    K, N = 192, 72
    g = torch.Generator(device=DEV)
    g.manual_seed(13)
    x, w, _, _, x64, w64 = operands("bf16", M, N, K, g)
    buffer = torch.zeros((M, K + N), dtype=torch.bfloat16, device=DEV)
    buffer[:, :K] = x
    gc.gc_linear(buffer[:, :K], w, out=buffer[:, K:])
    check(buffer[:, K:], *expected(x64, w64, None, "none", False, None, False))
    assert torch.equal(buffer[:, :K], x)
    with pytest.raises(gc.GeoCacheError, match="overlaps x"):
        gc.gc_linear(buffer[:, :K], w, out=buffer[:, K - 8:-8])


@pytest.mark.parametrize("kind,out", PAIRS)
@pytest.mark.parametrize("M", [3, 90, 600])
def test_weight_rows_that_repeat(gc, kind, out, M):
    g = torch.Generator(device=DEV)
    g.manual_seed(14)
    x, w, xs, ws, x64, w64 = operands(kind, M, 1, 272, g)
    got = gc.gc_linear(x, w.expand(150, -1), x_scale=xs, w_scale=None if ws is None else ws.expand(150).contiguous(),
                       out_dtype=TYPES[out])
    check(got, *expected(x64, w64.expand(150, -1), None, "none", False, None, kind == "e4m3" and out == "bf16"))
    assert bool((got == got[:, :1]).all())


@pytest.mark.parametrize("kind,M", [("bf16", 3), ("bf16", 40), ("f32", 2), ("f32", 40), ("e4m3", 20)])
def test_the_longest_rows(gc, kind, M):
    K, N, out = 1 << 20, 20, "f32"
    g = torch.Generator(device=DEV)
    g.manual_seed(15)
    x, w, xs, ws, x64, w64 = operands(kind, M, N, K, g)
    got = gc.gc_linear(x, w, x_scale=xs, w_scale=ws, out_dtype=TYPES[out])
    want = x64 @ w64.t()
    # (K u S would say nothing here: the products' signs are random, and the error is within 64 sqrt(K) u of their root)
    root = (x64.square() @ w64.square().t()).sqrt()
    assert float(((got.double() - want).abs() / root).max()) < 64 * math.sqrt(K) * U


def test_the_widest_output(gc):
    g = torch.Generator(device=DEV)
    g.manual_seed(16)
    for M in (2, 33):
        x, w, _, _, x64, w64 = operands("bf16", M, 300001, 16, g)
        got = gc.gc_linear(x, w, act=1)
        check(got, *expected(x64, w64, None, "silu", False, None, False))


def test_more_rows_than_a_launch_has_tiles(gc):
    """Rows past one launch's tiles go out in the next one."""
    M, N, K = (1 << 26) + 100003, 8, 4
    x = torch.randint(-4, 5, (M, K), device=DEV, dtype=torch.int8).float()
    w = torch.randint(-4, 5, (N, K), device=DEV, dtype=torch.int8).float()
    r = torch.randint(-4, 5, (M, 1), device=DEV, dtype=torch.int8).float().expand(-1, N).contiguous()
    got = gc.gc_linear(x, w, residual=r, out=r)
    first = r is got
    for i in (0, (1 << 26) - 70, M - 1000):
        n = min(1000, M - i)
        part = got[i:i + n] - x[i:i + n] @ w.t()
        assert bool((part == part[:, :1]).all()) and bool((part.abs() <= 4).all())   # whole numbers: exact
    assert first
    del x, r, got
    torch.cuda.empty_cache()
