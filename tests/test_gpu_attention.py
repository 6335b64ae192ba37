"""Attention over packed sequences against the formula in float64.

Tolerance, from the arithmetic.  With e = 2^-24: a score's error is at most
(dim + 4) e scale sum |q||k| (float32 products and sums of exact inputs, one
multiplication by the scale); an exponential adds 4 e relative and the
exponent's own rounding, at most 2^-23 |s - max|; sums of n terms add n e
relative; bfloat16 heads round each weight once more, by at most 2^-8
relative.  With d the largest score error and A = sum p |v| / sum p,
  |out - exact| <= (2 d + 2^-23 * 2 span + (n + 16) e [+ 2^-8]) A + rounding of out,
  |lse - exact| <= d + 2^-22 span + (n + 16) e + 2^-23 |lse|,
where span is the range of the row's scores.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def make(q_lens, k_lens, H, Hk, D, dtype, seed=1, spread=1.0):
    g = gen(seed)
    q = (torch.randn((sum(q_lens), H, D), generator=g, device=DEV) * spread).to(dtype)
    k = torch.randn((sum(k_lens), Hk, D), generator=g, device=DEV).to(dtype)
    v = (torch.randn((sum(k_lens), Hk, D), generator=g, device=DEV) + 0.3).to(dtype)
    return q, k, v


def reference(q, k, v, q_lens, k_lens, causal, scale):
    """(out, lse, bound of out, bound of lse), in float64, row by row of the mask."""
    T, H, D = q.shape
    G = H // max(1, k.shape[1])
    out = torch.zeros((T, H, D), dtype=torch.float64, device=DEV)
    lse = torch.full((H, T), -math.inf, dtype=torch.float64, device=DEV)
    tol_o = torch.full((T, H, D), 2.0 ** -120, dtype=torch.float64, device=DEV)
    tol_l = torch.full((H, T), 2.0 ** -120, dtype=torch.float64, device=DEV)
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        if nq and nk:
            seen = torch.ones((nq, nk), dtype=torch.bool, device=DEV)
            if causal:
                seen = torch.arange(nk, device=DEV) <= torch.arange(nq, device=DEV)[:, None] + nk - nq
            for h in range(H):
                Q, K, V = (t.double().contiguous() for t in (q[q0:q0 + nq, h], k[k0:k0 + nk, h // G], v[k0:k0 + nk, h // G]))
                s = (Q @ K.t().contiguous() * scale).masked_fill(~seen, -math.inf)
                d = ((Q.abs() @ K.abs().t().contiguous()) * scale * (D + 4) * E).masked_fill(~seen, 0).amax(-1)
                m = s.amax(-1, keepdim=True)
                some = (m > -math.inf)[:, 0]
                p = torch.exp(s - torch.where(m > -math.inf, m, 0.0))
                span = torch.where(seen & (p > 0), (m - s).abs(), 0.0).amax(-1)
                l = p.sum(-1, keepdim=True).clamp_min(1e-300)
                o, A = p @ V / l, p @ V.abs() / l
                rel = 2 * d + 2.0 ** -22 * span + (nk + 16) * E + (2.0 ** -8 if q.dtype == BF16 else 0)
                out[q0:q0 + nq, h] = torch.where(some[:, None], o, 0.0)
                tol_o[q0:q0 + nq, h] += rel[:, None] * A + (2.0 ** -8 * 1.01 * o.abs() if q.dtype == BF16 else 2 * E * o.abs())
                e = torch.where(some, m[:, 0] + l[:, 0].log(), -math.inf)
                lse[h, q0:q0 + nq] = e
                tol_l[h, q0:q0 + nq] += torch.where(some, d + 2.0 ** -22 * span + (nk + 16) * E + 2.0 ** -23 * e.abs(), 0.0)
        q0, k0 = q0 + nq, k0 + nk
    return out, lse, tol_o, tol_l


def check(got, want):
    out, lse = got
    o, e, to, tl = want
    bad = ~((out.double() - o).abs() <= to)
    assert not bad.any(), (f"out: {int(bad.sum())} of {bad.numel()} beyond the bound, first at "
                           f"{bad.nonzero()[0].tolist()}, worst {float(((out.double() - o).abs() / to).nan_to_num(9e9).max()):.3g} x")
    empty = e == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    bad = ~((lse.double() - e).abs() <= tl) & ~empty
    assert not bad.any(), f"lse: {int(bad.sum())} of {bad.numel()} beyond the bound, first at {bad.nonzero()[0].tolist()}"


def run(gc, q_lens, k_lens, H, Hk, D, dtype, causal, scale=None, seed=1, spread=1.0):
    q, k, v = make(q_lens, k_lens, H, Hk, D, dtype, seed, spread)
    plan = gc.gc_attention_plan(q_lens, k_lens, H, Hk, D, dtype, causal=causal, device=DEV)
    got = gc.gc_attention(q, k, v, plan, scale=scale)
    check(got, reference(q, k, v, q_lens, k_lens, causal, 1 / math.sqrt(D) if scale is None else scale))
    # the same again, bit for bit (the workspace is ready for the next call)
    again = gc.gc_attention(q, k, v, plan, scale=scale)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
CAUSAL = pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])

LENS = [
    ([1], [1]),
    ([1, 2, 3], [1, 2, 3]),
    ([63, 64, 65], [63, 64, 65]),
    ([127, 0, 129, 1], [127, 5, 129, 1]),              # a sequence without queries
    ([5, 3, 2], [0, 3, 70]),                           # one without keys
    ([300], [300]),
    ([31, 40], [7, 200]),                              # more queries than keys, and fewer
    ([100, 1], [333, 1000]),
]


@DTYPES
@CAUSAL
@pytest.mark.parametrize("q_lens,k_lens", LENS)
def test_lengths(gc, q_lens, k_lens, causal, dtype):
    run(gc, q_lens, k_lens, 4, 2, 64, dtype, causal)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [8, 24, 32, 40, 64, 72, 80, 96, 104, 128, 136, 160, 192, 200, 256])
def test_dims(gc, D, causal, dtype):
    run(gc, [70, 33, 1], [70, 150, 9], 4, 4, D, dtype, causal, seed=D)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("H,Hk", [(1, 1), (3, 3), (6, 2), (8, 1), (7, 1), (64, 8), (5, 5), (40, 2)])
def test_groups(gc, H, Hk, causal, dtype):
    run(gc, [45, 1, 12], [90, 77, 12], H, Hk, 64, dtype, causal, seed=H)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("H,Hk,D", [(32, 8, 128), (8, 8, 64), (16, 1, 80), (2, 2, 256)])
@pytest.mark.parametrize("k_lens", [[1, 63, 64, 65, 1000], [5000], [33, 20000, 129, 1]], ids=["short", "one", "long"])
def test_single_tokens(gc, k_lens, H, Hk, D, causal, dtype):
    """One query token a sequence over its kept keys."""
    run(gc, [1] * len(k_lens), k_lens, H, Hk, D, dtype, causal, seed=3)


@DTYPES
@pytest.mark.parametrize("q_lens", [[2], [5, 3], [17], [40]], ids=str)
def test_few_tokens_over_many_keys(gc, q_lens, dtype):
    run(gc, q_lens, [9001] * len(q_lens), 8, 2, 128, dtype, True, seed=4)


@DTYPES
@CAUSAL
def test_many_sequences(gc, causal, dtype):
    lens = [(7 * i * i + 3 * i) % 91 for i in range(150)]
    run(gc, lens, [n + (i % 3) * 17 for i, n in enumerate(lens)], 4, 1, 64, dtype, causal, seed=5)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [64, 128])
def test_longer(gc, D, causal, dtype):
    run(gc, [2049, 700, 1], [2049, 1500, 3], 4, 2, D, dtype, causal, seed=6)


@DTYPES
def test_large_scores_and_scales(gc, dtype):
    """Weights that concentrate on few keys, rows whose maximum keeps growing along the keys."""
    run(gc, [200], [500], 2, 2, 64, dtype, False, spread=30.0, seed=7)
    run(gc, [200], [500], 2, 2, 64, dtype, True, scale=0.001, seed=7)
    q, k, v = make([64], [640], 2, 2, 64, dtype, 8)
    ramp = torch.linspace(0.1, 6.0, 640, device=DEV)[:, None, None]
    q = q.abs()
    k = (k.abs() * ramp).to(dtype)
    plan = gc.gc_attention_plan([64], [640], 2, 2, 64, dtype, device=DEV)
    check(gc.gc_attention(q, k, v, plan), reference(q, k, v, [64], [640], False, 0.125))


@DTYPES
@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf], ids=str)
def test_masked_places_have_no_effect(gc, bad, D, dtype):
    """Keys and values that a causal row does not see, and the tokens of the
    next sequence, hold NaN or infinity: rows that see none of it are as
    without it, bit for bit."""
    q_lens, k_lens, H = [150, 40, 1], [150, 300, 64], 2
    q, k, v = make(q_lens, k_lens, H, H, D, dtype, 9)
    plan = gc.gc_attention_plan(q_lens, k_lens, H, H, D, dtype, causal=True, device=DEV)
    clean, clean_l = gc.gc_attention(q, k, v, plan)
    k2, v2 = k.clone(), v.clone()
    k2[100, :, 3] = bad           # seen by queries 100.. of the first sequence
    v2[100, :, 5] = bad
    v2[101] = bad
    k2[150 + 290, 0] = bad        # seen by the second sequence's last queries
    v2[150 + 290, 0] = bad
    got, lse = gc.gc_attention(q, k2, v2, plan)
    rows = list(range(100)) + list(range(150, 150 + 30)) + [190]
    assert torch.equal(got[rows], clean[rows]) and torch.equal(lse[:, rows], clean_l[:, rows])
    # the second head sees nothing of the second sequence's
    assert torch.equal(got[150:, 1], clean[150:, 1])
    # rows that see a value of NaN or infinity say so
    assert not got[101, :].isfinite().all()
    assert bool((~got[101:150].isfinite()).any(-1).all())


@DTYPES
def test_padding_channels_and_next_tokens(gc, dtype):
    """A head of 72 channels inside a wider buffer whose other channels, and
    the tokens after the last, hold NaN."""
    D, H = 72, 2
    q_lens, k_lens = [50, 9], [50, 77]
    q, k, v = make(q_lens, k_lens, H, H, D, dtype, 10)
    plan = gc.gc_attention_plan(q_lens, k_lens, H, H, D, dtype, device=DEV)
    want = gc.gc_attention(q, k, v, plan)

    def wrap(t):
        big = torch.full((t.shape[0] + 40, H + 1, 104), math.nan, dtype=dtype, device=DEV)
        big[:t.shape[0], :H, 8:8 + D] = t
        return big[:t.shape[0], :H, 8:8 + D]

    got = gc.gc_attention(wrap(q), wrap(k), wrap(v), plan, out=wrap(torch.zeros_like(q)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@DTYPES
@CAUSAL
def test_scores_of_minus_infinity(gc, causal, dtype):
    """Every score of a row -inf (keys of -inf against positive queries): a
    row as without keys; NaN queries give NaN rows and no others."""
    q, k, v = make([70], [70], 2, 2, 64, dtype, 11)
    q = q.abs() + 0.1
    plan = gc.gc_attention_plan([70], [70], 2, 2, 64, dtype, causal=causal, device=DEV)
    k2 = k.clone()
    k2[:, 0] = -math.inf
    out, lse = gc.gc_attention(q.to(dtype), k2, v, plan)
    assert not out[:, 0].any() and bool((lse[0] == -math.inf).all())
    assert bool(out[:, 1].isfinite().all())
    clean, _ = gc.gc_attention(q.to(dtype), k, v, plan)
    q2 = q.to(dtype).clone()
    q2[13, 1] = math.nan
    out, lse = gc.gc_attention(q2, k, v, plan)
    assert bool(out[13, 1].isnan().all()) and bool(lse[1, 13].isnan())
    keep = [i for i in range(70) if i != 13]
    assert torch.equal(out[keep], clean[keep]) and torch.equal(out[13, 0], clean[13, 0])


@DTYPES
def test_strides(gc, dtype):
    """Columns of a fused projection, heads before tokens, broadcast keys."""
    H, Hk, D, n = 6, 2, 64, [130, 75]
    q, k, v = make(n, n, H, Hk, D, dtype, 12)
    plan = gc.gc_attention_plan(n, n, H, Hk, D, dtype, causal=True, device=DEV)
    want = gc.gc_attention(q, k, v, plan)
    fused = torch.cat([q, k, v], 1).contiguous()
    got = gc.gc_attention(*fused.split([H, Hk, Hk], 1), plan)
    assert torch.equal(got[0], want[0])
    hf = [t.permute(1, 0, 2).contiguous().permute(1, 0, 2) for t in (q, k, v)]
    out = torch.empty((H, sum(n), D), dtype=dtype, device=DEV).permute(1, 0, 2)
    assert torch.equal(gc.gc_attention(*hf, plan, out=out)[0], want[0])
    one = gc.gc_attention(q, k[:, :1].expand(-1, Hk, -1), v[:, :1].expand(-1, Hk, -1), plan)[0]
    both = gc.gc_attention(q, k[:, :1].repeat(1, Hk, 1), v[:, :1].repeat(1, Hk, 1), plan)[0]
    assert torch.equal(one, both)


@DTYPES
def test_offsets_past_32_bits(gc, dtype):
    """Kept keys 2^20 elements apart: byte offsets pass 2^32, for single tokens and for many."""
    S, D = 3000, 64
    big = torch.empty((S, 1 << 20), dtype=dtype, device=DEV)
    k, v = big[:, 64:128].unsqueeze(1), big[:, 1024:1088].unsqueeze(1)
    for n in (1, 200):
        q, k0, v0 = make([n], [S], 2, 1, D, dtype, 13)
        k.copy_(k0), v.copy_(v0)
        plan = gc.gc_attention_plan([n], [S], 2, 1, D, dtype, causal=True, device=DEV)
        want = gc.gc_attention(q, k0, v0, plan)
        got = gc.gc_attention(q, k, v, plan)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@DTYPES
def test_sequences_do_not_depend_on_their_neighbours_values(gc, dtype):
    """A packed batch equals the same batch with other tokens elsewhere."""
    lens = [90, 1, 260]
    q, k, v = make(lens, lens, 4, 4, 64, dtype, 14)
    plan = gc.gc_attention_plan(lens, lens, 4, 4, 64, dtype, device=DEV)
    a = gc.gc_attention(q, k, v, plan)[0]
    k2, v2 = k.clone(), v.clone()
    k2[:90], v2[91:] = 7.0, -3.0
    b = gc.gc_attention(q, k2, v2, plan)[0]
    assert torch.equal(a[90:91], b[90:91])


def test_nothing_to_do(gc):
    for q_lens, k_lens in (([], []), ([0, 0], [5, 0])):
        plan = gc.gc_attention_plan(q_lens, k_lens, 4, 2, 64, BF16, device=DEV)
        k = torch.zeros((sum(k_lens), 2, 64), dtype=BF16, device=DEV)
        out, lse = gc.gc_attention(torch.empty((0, 4, 64), dtype=BF16, device=DEV), k, k, plan)
        assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    plan = gc.gc_attention_plan([3], [0], 4, 2, 64, F32, device=DEV)       # queries, and no key anywhere
    none = torch.empty((0, 2, 64), device=DEV)
    out, lse = gc.gc_attention(torch.randn((3, 4, 64), device=DEV), none, none, plan)
    assert not out.any() and bool((lse == -math.inf).all())


@DTYPES
def test_streams_with_plans_of_their_own(gc, dtype):
    k_lens, H, Hk, D = [20000, 300, 5], 16, 4, 128
    q, k, v = make([1] * 3, k_lens, H, Hk, D, dtype, 15)
    plan = gc.gc_attention_plan([1] * 3, k_lens, H, Hk, D, dtype, device=DEV)
    want = gc.gc_attention(q, k, v, plan)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    plans = [gc.gc_attention_plan([1] * 3, k_lens, H, Hk, D, dtype, device=DEV, stream=s) for s in streams]
    got = [gc.gc_attention(q, k, v, p, stream=s) for _ in range(5) for s, p in zip(streams, plans)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) and torch.equal(e, want[1]) for o, e in got)


@DTYPES
def test_graph_replays(gc, dtype):
    """A captured call, replayed over changing inputs with eager work between
    the replays, equals the eager call each time."""
    k_lens, H, Hk, D = [5000, 64], 8, 2, 64
    q, k, v = make([1, 30], k_lens, H, Hk, D, dtype, 16)
    plan = gc.gc_attention_plan([1, 30], k_lens, H, Hk, D, dtype, causal=True, device=DEV)
    out, lse = torch.empty_like(q), torch.empty((H, 31), device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        gc.gc_attention(q, k, v, plan, out=out, lse=lse)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gc.gc_attention(q, k, v, plan, out=out, lse=lse)
    for i in range(4):
        fresh = make([1, 30], k_lens, H, Hk, D, dtype, 20 + i)
        for t, f in zip((q, k, v), fresh):
            t.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        want = gc.gc_attention(*fresh, plan)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_more_blocks_than_a_launch_has_threads_for(gc):
    """600000 sequences of one token and one key: every result is its value, past the first launch's too."""
    n, H, D = 600000, 16, 32
    g = gen(41)
    q, k, v = (torch.randn((n, H, D), generator=g, device=DEV).bfloat16() for _ in range(3))
    plan = gc.gc_attention_plan([1] * n, [1] * n, H, H, D, torch.bfloat16, causal=True, device=DEV)
    assert torch.equal(gc.gc_attention(q, k, v, plan)[0], v)
