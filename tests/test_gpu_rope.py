"""Rotary positions and the per-head norms with the rotation, against the
formulas in float64.

Tolerance, from the arithmetic: a turned channel is a c - b s in float32 from
exact inputs (two products, one sum), so its error is at most 3 * 2^-24
(|a| + |b|) with |c|, |s| <= 1; the norm's factor r adds a relative error of
at most (dim/8 + 8) * 2^-24 (the lanes' sums of at most dim/lanes squares, the butterfly,
the mean, the root and the division), the gain one more rounding.  A bfloat16 store rounds by at most
2^-8 of the value.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def turn64(x, positions, table, sections, layout):
    """x float64 [T, heads, D] turned, and the sum |a| + |b| of each channel's pair."""
    half = sum(sections)
    pos = positions.reshape(x.shape[0], -1)
    cols = torch.cat([torch.full((n,), a) for a, n in enumerate(sections)]).to(DEV)
    t = table.double()
    at = pos[:, cols].long()
    cs = t[at.clamp(0, t.shape[0] - 1), torch.arange(half, device=DEV)]
    cs = torch.where(((at < 0) | (at >= t.shape[0]))[..., None], math.nan, cs)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    ia = torch.arange(half, device=DEV) if layout == 0 else 2 * torch.arange(half, device=DEV)
    ib = ia + half if layout == 0 else ia + 1
    y, mag = x.clone(), x.abs()
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia] = mag[..., ib] = a.abs() + b.abs()
    return y, mag


def close(got, want, mag, rel, dtype):
    tol = rel * mag + (want.abs() * 2.0 ** -8 * (1 + 2.0 ** -8) if dtype == torch.bfloat16 else 0) + 2.0 ** -133
    bad = ~((got.double() - want).abs() <= tol) & ~(got.isnan() & want.isnan())
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} beyond the bound, first at {bad.nonzero()[0].tolist()}"


def table_for(gc, n_pos, sections):
    return gc.gc_rope_table(n_pos, sections, device=DEV)


CASES = [  # T, H, D, sections
    (1, 1, 8, [2]), (1, 32, 128, [64]), (3, 5, 64, [8, 12, 12]), (257, 3, 72, [9, 13, 14]), (100, 4, 80, [4, 8, 8]),
    (33, 7, 96, [24]), (65, 2, 192, [96]), (129, 1, 256, [32, 48, 48]), (31, 9, 40, [1, 1]), (7, 70, 128, [10, 11, 12, 13]),
    (1000, 16, 64, [16]), (5, 3, 72, [36]), (64, 2, 16, [4]),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1], ids=["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,sections", CASES)
def test_rope(gc, T, H, D, sections, layout, dtype):
    g = gen(T + H)
    x = torch.randn((T, H, D), generator=g, device=DEV).to(dtype)
    pos = torch.randint(0, 5000, (T, len(sections)), generator=g, device=DEV).int()
    table = table_for(gc, 5000, sections)
    y, mag = turn64(x.double(), pos, table, sections, layout)
    keep = x.clone()
    got = gc.gc_rope(x, pos, table, sections, layout)
    close(got, y, mag, 3 * U, dtype)
    assert torch.equal(x, keep)
    assert torch.equal(got[..., 2 * sum(sections):], x[..., 2 * sum(sections):])
    same = gc.gc_rope(x, pos, table, sections, layout, out=x)          # in place
    assert same is x and torch.equal(x, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1], ids=["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,sections", CASES)
def test_qk_norm_rope(gc, T, H, D, sections, layout, dtype):
    g = gen(T + 7 * H)
    Hk = max(1, H // 2)
    # columns of one fused projection, a large and a small magnitude among the tokens
    full = torch.randn((T, H + 2 * Hk, D), generator=g, device=DEV)
    full[::3] *= 1e-4
    full[1::5] *= 1e4
    full = full.to(dtype)
    q, k, _ = full.split([H, Hk, Hk], dim=1)
    gq, gk = (torch.randn((D,), generator=g, device=DEV) for _ in range(2))
    pos = torch.randint(0, 300, (T, len(sections)), generator=g, device=DEV).int()
    table = table_for(gc, 300, sections)
    want = []
    for x, gain in ((q, gq), (k, gk)):
        x = x.double()
        want.append(turn64(x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain.double(), pos, table, sections, layout))
    rest = full[:, H + Hk:].clone()
    got = gc.gc_qk_norm_rope(q, k, gq, gk, pos, table, sections=sections, layout=layout)
    for y, (w, mag) in zip(got, want):
        close(y, w, mag, (D / 8 + 14) * U, dtype)
    again = gc.gc_qk_norm_rope(q, k, gq, gk, pos, table, sections=sections, layout=layout, q_out=q, k_out=k)
    assert torch.equal(q, got[0]) and torch.equal(k, got[1]) and again[0] is q
    assert torch.equal(full[:, H + Hk:], rest)


def test_heads_first_order_and_a_wide_stride(gc):
    g = gen(5)
    T, H, D, sec = 77, 6, 64, [32]
    table = table_for(gc, 100, sec)
    pos = torch.randint(0, 100, (T,), generator=g, device=DEV).int()
    x = torch.randn((T, H, D), generator=g, device=DEV)
    want = gc.gc_rope(x, pos, table)
    heads_first = x.permute(1, 0, 2).contiguous().permute(1, 0, 2)
    out = torch.empty((H, T, D), device=DEV).permute(1, 0, 2)
    assert torch.equal(gc.gc_rope(heads_first, pos, table, out=out), want)
    wide = torch.zeros((T, H, 200), device=DEV)
    wide[..., 96:160] = x
    assert torch.equal(gc.gc_rope(wide[..., 96:160], pos, table), want)


def test_positions_outside_the_table_give_nan(gc):
    x = torch.ones((3, 2, 16), device=DEV)
    table = table_for(gc, 10, [2, 2])
    pos = torch.tensor([[9, 0], [10, 3], [2, -1]], dtype=torch.int32, device=DEV)
    y = gc.gc_rope(x, pos, table, [2, 2])
    nan = y[:, 0].isnan()
    assert not nan[0].any() and not nan[:, 8:].any()
    assert nan[1].nonzero().flatten().tolist() == [0, 1, 4, 5]
    assert nan[2].nonzero().flatten().tolist() == [2, 3, 6, 7]


def test_nan_and_infinity_stay_in_their_head(gc):
    g = gen(6)
    T, H, D = 9, 4, 64
    q = torch.randn((T, H, D), generator=g, device=DEV)
    k = torch.randn((T, H, D), generator=g, device=DEV)
    gain = torch.ones(D, device=DEV)
    pos = torch.arange(T, device=DEV).int()
    table = table_for(gc, T, [32])
    clean = gc.gc_qk_norm_rope(q, k, gain, gain, pos, table)
    q[2, 1, 5] = math.nan
    k[3, 2, 60] = math.inf
    got = gc.gc_qk_norm_rope(q, k, gain, gain, pos, table)
    for c, y, (t, h) in ((clean[0], got[0], (2, 1)), (clean[1], got[1], (3, 2))):
        assert y[t, h].isnan().any()
        mask = torch.ones((T, H), dtype=torch.bool, device=DEV)
        mask[t, h] = False
        assert torch.equal(c[mask], y[mask])


def test_rows_of_zeros(gc):
    z = torch.zeros((2, 1, 32), device=DEV)
    gain = torch.ones(32, device=DEV)
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    q, k = gc.gc_qk_norm_rope(z, z, gain, gain, pos, table_for(gc, 1, [16]))
    assert not q.any() and not k.any()


def test_no_tokens(gc):
    e = torch.empty((0, 4, 64), device=DEV)
    pos = torch.empty((0, 1), dtype=torch.int32, device=DEV)
    table = table_for(gc, 4, [32])
    gain = torch.ones(64, device=DEV)
    assert gc.gc_rope(e, pos, table).shape == (0, 4, 64)
    assert [t.shape[0] for t in gc.gc_qk_norm_rope(e, e, gain, gain, pos, table)] == [0, 0]


@pytest.mark.parametrize("scaling", [None, (4.0, 8192.0, 1.0, 4.0, 1.0), (32.0, 4096.0, 1.0, 32.0, 1.3466),
                                     (8.0, 2048.0, math.inf, math.inf, 1.0), (2.0, 1000.0, 3.0, 3.0, 1.0)])
def test_table(gc, scaling):
    """cos and sin of p f in double, rounded once: half an ulp of float32,
    and the angle's own double rounding, which grows with it."""
    sections, base, n_pos = [16, 24, 8], 500000.0, 70000
    sc = None if scaling is None else gc.RopeScaling(*scaling)
    got = gc.gc_rope_table(n_pos, sections, base, sc, device=DEV).double().cpu()
    f = torch.cat([torch.tensor([base ** (-i / n) for i in range(n)], dtype=torch.float64) for n in sections])
    amp = 1.0
    if scaling is not None:
        s, L0, lo, hi, amp = scaling
        r = L0 * f / (2 * math.pi)
        gmix = ((r - lo) / (hi - lo)).clamp(0, 1) if hi > lo else (r >= lo).double()
        f = gmix * f + (1 - gmix) * f / s
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * f
    want = amp * torch.stack([angle.cos(), angle.sin()], -1)
    tol = want.abs() * 2.0 ** -24 * (1 + 2.0 ** -10) + amp * (angle[..., None] * 2.0 ** -50 + 2.0 ** -48)
    assert bool(((got - want).abs() <= tol).all())


def test_a_stream_of_its_own(gc):
    g = gen(8)
    x = torch.randn((4096, 16, 128), generator=g, device=DEV).bfloat16()
    pos = torch.arange(4096, device=DEV).int()
    table = table_for(gc, 4096, [64])
    want = gc.gc_rope(x, pos, table)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [gc.gc_rope(x, pos, table, stream=s) for _ in range(4)]
    s.synchronize()
    assert all(torch.equal(y, want) for y in got)


def test_offsets_past_32_bits(gc):
    """Tokens two million elements apart: byte offsets pass 2^32."""
    T, D = 1100, 64
    big = torch.empty((T, 1 << 21), dtype=torch.bfloat16, device=DEV)
    view = big[:, 512:512 + D].unsqueeze(1)
    x = torch.randn((T, 1, D), generator=gen(9), device=DEV).bfloat16()
    view.copy_(x)
    pos = torch.arange(T, device=DEV).int()
    table = table_for(gc, T, [32])
    want = gc.gc_rope(x, pos, table)
    assert torch.equal(gc.gc_rope(view, pos, table), want)
    gc.gc_rope(view, pos, table, out=view)
    assert torch.equal(view, want)


def test_more_tokens_than_a_launch_has_threads_for(gc):
    """2^25 + 40 heads of 64 lanes each: over 2^31 threads, tokens past the first launch's among them."""
    T, D = (1 << 25) + 40, 256
    x = torch.zeros((T, 1, D), dtype=torch.bfloat16, device=DEV)
    rows = torch.tensor([0, 1, T // 2, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, T - 1], device=DEV)
    x[rows] = torch.randn((rows.numel(), 1, D), generator=gen(11), device=DEV).bfloat16()
    pos = torch.arange(T, device=DEV).remainder_(64).int()
    table = table_for(gc, 64, [2])
    want = gc.gc_rope(x[rows], pos[rows].contiguous(), table)
    gc.gc_rope(x, pos, table, out=x)
    assert torch.equal(x[rows], want)
    assert int(torch.count_nonzero(x.view(T, D).any(dim=1))) == rows.numel()


@pytest.mark.parametrize("eps", [1e-45, 1e-30, 1e-6])
def test_rows_of_zeros_with_a_small_eps(gc, eps):
    z = torch.zeros((2, 1, 32), device=DEV)
    gain = torch.ones(32, device=DEV)
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    q, k = gc.gc_qk_norm_rope(z, z, gain, gain, pos, table_for(gc, 1, [16]), eps=eps)
    assert torch.equal(q, z) and torch.equal(k, z)
