"""Values of infinity and NaN that a row sees.

A channel in which a row sees a value that is not finite holds the sum of
those values (an infinity, or NaN for NaN and for infinities of both signs),
however small their weights: not 0 times infinity where a weight underflows,
whatever tiles, parts and waves the keys are dealt to.  Every other channel is
as without them, within the bounds of the operator's arithmetic.
"""
import math

import pytest
import torch

from test_gpu_attention import BF16, DEV, F32, check, gen, reference

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


# lengths, heads, kv heads, dim, type, causal; the variant and whether keys are split, as the plan has it
FORMS = {
    "keys": ([5, 1], [300, 77], 8, 2, 64, BF16, False, 2, False),
    "keys_split": ([5, 1], [300, 9000], 8, 2, 64, BF16, True, 2, True),
    "keys_f32": ([5], [300], 8, 2, 32, F32, True, 2, False),
    "keys_f32_split": ([32], [2000], 1, 1, 80, F32, False, 2, True),
    "keys_wide": ([5, 2], [300, 5000], 4, 1, 192, BF16, True, 2, True),
    "rows": ([200, 70], [640, 300], 2, 2, 64, BF16, False, 1, False),
    "rows_causal": ([200, 70], [640, 300], 2, 2, 128, BF16, True, 1, False),
    "rows_wide": ([200, 70], [640, 300], 2, 2, 200, BF16, True, 1, True),
    "rows_f32": ([256] * 16, [640] * 16, 16, 16, 64, F32, True, 1, False),
    "rows_f32_split": ([200, 70], [640, 300], 2, 2, 72, F32, False, 1, True),
    "rows_256": ([256] * 16, [640] * 16, 16, 16, 64, BF16, True, 0, False),
    "rows_256_split": ([3000], [3000], 4, 4, 128, BF16, False, 0, True),
}


def ramp(nk, order):
    """Scores that fall, or rise, by 400 along the keys: most weights underflow."""
    r = torch.linspace(-20.0, 0.0, nk, device=DEV)
    return r.flip(0) if order == "falling" else r


@pytest.mark.parametrize("order", ["falling", "rising", "flat"])
@pytest.mark.parametrize("form", FORMS)
def test_seen_values_that_are_not_finite(gc, form, order):
    q_lens, k_lens, H, Hk, D, dtype, causal, kind, split = FORMS[form]
    plan = gc.gc_attention_plan(q_lens, k_lens, H, Hk, D, dtype, causal=causal, device=DEV)
    assert plan.info.kind == kind and (plan.info.n_slots > 0) == split
    g = gen(31)
    q = torch.randn((sum(q_lens), H, D), generator=g, device=DEV) * 0.1
    k = torch.randn((sum(k_lens), Hk, D), generator=g, device=DEV)
    v = torch.randn((sum(k_lens), Hk, D), generator=g, device=DEV)
    if order != "flat":
        q[..., 0] = 20.0
        k[..., 0] = torch.cat([ramp(n, order) for n in k_lens])[:, None]
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    bad = v.clone()
    k0 = 0
    for n in k_lens:
        places = sorted({0, 3, n // 7, n // 3, n // 2, 2 * n // 3, max(0, n - 70), n - 2, n - 1})
        for i, j in enumerate(places):
            bad[k0 + j, :, (3 * i + 1) % D] = (INF, -INF, NAN)[i % 3]
            bad[k0 + j, :, D - 2] = INF                       # a channel of infinities of one sign
        bad[k0 + n // 5, 0, D - 3], bad[k0 + n - 1, 0, D - 3] = INF, -INF     # of both
        k0 += n
    scale = 1.0
    out, lse = gc.gc_attention(q, k, bad, plan, scale=scale)
    again = gc.gc_attention(q, k, bad, plan, scale=scale)
    same = lambda a, b: torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    assert same(out, again[0]) and torch.equal(lse, again[1])

    # what each row sees that is not finite, summed: as numbers of +inf, -inf and NaN
    G = H // Hk
    kinds = [(bad == INF).float(), (bad == -INF).float(), bad.isnan().float()]
    counts = [torch.zeros((sum(q_lens), H, D), device=DEV) for _ in kinds]
    q0 = k0 = 0
    for nq, nk in zip(q_lens, k_lens):
        seen = torch.ones((nq, nk), device=DEV)
        if causal:
            seen = (torch.arange(nk, device=DEV) <= torch.arange(nq, device=DEV)[:, None] + nk - nq).float()
        for which, c in zip(kinds, counts):
            for h in range(H):
                c[q0:q0 + nq, h] = seen @ which[k0:k0 + nk, h // G].contiguous()
        q0, k0 = q0 + nq, k0 + nk
    up, down, nan = (c > 0 for c in counts)
    want_nan = nan | (up & down)
    touched = up | down | nan
    assert torch.equal(out.isnan(), want_nan)
    assert torch.equal(out == INF, up & ~want_nan) and torch.equal(out == -INF, down & ~want_nan)
    # the other channels, and the log-sum-exp
    clean = torch.where(bad.isfinite(), bad, torch.zeros_like(bad))
    o, e, to, tl = reference(q, k, clean, q_lens, k_lens, causal, scale)
    got = torch.where(touched, torch.zeros_like(out), out)
    check((got, lse), (torch.where(touched, 0.0, o), e, to, tl))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("q_lens,k_lens", [([3], [500]), ([90], [500]), ([2], [9000])], ids=str)
def test_rows_of_nan_scores_stay_nan(gc, q_lens, k_lens, dtype):
    """A query of NaN, or a key of NaN that a row sees, makes all of the row's channels NaN, those with infinite values too."""
    g = gen(32)
    q, k, v = (torch.randn((n, 2, 64), generator=g, device=DEV).to(dtype) for n in (sum(q_lens), sum(k_lens), sum(k_lens)))
    v[7, :, 5], v[400, :, 9] = INF, -INF
    q[1, 0, 3] = NAN
    plan = gc.gc_attention_plan(q_lens, k_lens, 2, 2, 64, dtype, device=DEV)
    out, lse = gc.gc_attention(q, k, v, plan)
    assert bool(out[1, 0].isnan().all()) and bool(lse[0, 1].isnan())
    assert bool((out[1, 1, 5] == INF)) and bool((out[1, 1, 9] == -INF)) and not out[:, 1].isnan().any()
    k[450, 1, 0] = NAN
    out, lse = gc.gc_attention(q, k, v, plan)
    assert bool(out[:, 1].isnan().all()) and bool(lse[1].isnan().all()) and not out[0, 0].isnan().any()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("q_lens,k_lens", [([3], [500]), ([90], [500]), ([2], [9000])], ids=str)
def test_rows_without_a_finite_score_are_empty(gc, q_lens, k_lens, dtype):
    """Only scores of -inf: 0 and -inf, whatever the values."""
    g = gen(33)
    q = torch.randn((sum(q_lens), 2, 64), generator=g, device=DEV).abs().add(0.1).to(dtype)
    k, v = (torch.randn((sum(k_lens), 2, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    k[:, 0] = -INF
    v[7, :, 5], v[400, :, 9] = INF, NAN
    plan = gc.gc_attention_plan(q_lens, k_lens, 2, 2, 64, dtype, device=DEV)
    out, lse = gc.gc_attention(q, k, v, plan)
    assert not out[:, 0].any() and bool((lse[0] == -INF).all())
    assert bool((out[:, 1, 5] == INF).all()) and bool(out[:, 1, 9].isnan().all())
