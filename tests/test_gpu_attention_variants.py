"""Every kernel variant of the attention, at every padded head size, against
the formula in float64: the lengths are chosen so that the plan takes the
variant in question, with keys split and not, and so that a block walks from
one tile of keys to many with any remainder.  Bounds: those of the operator's
arithmetic (test_gpu_attention)."""
import math

import pytest
import torch

from test_gpu_attention import BF16, CAUSAL, DTYPES, F32, check, make, reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KEYS, ROWS128, ROWS256 = 2, 1, 0
NAN, INF = math.nan, math.inf

# numbers of keys: one tile of 64 to fifteen, whole and with remainders on either side of 32
TILES = [1, 40, 64, 65, 130, 191, 256, 300, 330, 385, 449, 513, 577, 640, 700, 901]
ONE_PER_TILE = {
    "rows256": ([256] * 16, TILES, 48, 16, ROWS256),
    "rows128": ([40] * 16, TILES, 2, 2, ROWS128),
    "keys": ([1, 2, 5] * 7, [31, 32, 33, 63, 65, 95, 97, 127, 128, 129, 160, 161, 191, 255, 256, 257, 300, 383, 385, 513, 640],
             4, 2, KEYS),
}
SPLIT = {
    "rows256": ([700, 650], [2700, 2650], 8, 2, ROWS256),
    "rows128": ([200, 70], [2640, 300], 2, 2, ROWS128),
    "keys": ([5, 1, 3], [300, 9000, 2001], 8, 2, KEYS),
}


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


def planned(gc, q_lens, k_lens, H, Hk, D, dtype, causal, kind, split=None):
    plan = gc.gc_attention_plan(q_lens, k_lens, H, Hk, D, dtype, causal=causal, device=DEV)
    assert plan.info.kind == kind
    assert split is None or (plan.info.n_slots > 0) == split
    return plan


def run(gc, q_lens, k_lens, H, Hk, D, dtype, causal, kind, split, seed):
    plan = planned(gc, q_lens, k_lens, H, Hk, D, dtype, causal, kind, split)
    q, k, v = make(q_lens, k_lens, H, Hk, D, dtype, seed)
    check(gc.gc_attention(q, k, v, plan), reference(q, k, v, q_lens, k_lens, causal, 1 / math.sqrt(D)))


@CAUSAL
@pytest.mark.parametrize("D", [8, 32, 40, 64, 80, 96, 104, 128])
def test_eight_waves_one_to_fifteen_tiles(gc, D, causal):
    q_lens, k_lens, H, Hk, kind = ONE_PER_TILE["rows256"]
    run(gc, q_lens, k_lens, H, Hk, D, BF16, causal, kind, False, D)


@CAUSAL
@pytest.mark.parametrize("D", [32, 64, 80, 128])
def test_eight_waves_split_keys(gc, D, causal):
    q_lens, k_lens, H, Hk, kind = SPLIT["rows256"]
    run(gc, q_lens, k_lens, H, Hk, D, BF16, causal, kind, True, D + 1)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [8, 32, 64, 96, 128, 192, 200, 256])
@pytest.mark.parametrize("form", ["rows128", "keys"])
def test_one_to_fifteen_tiles(gc, form, D, causal, dtype):
    q_lens, k_lens, H, Hk, kind = ONE_PER_TILE[form]
    run(gc, q_lens, k_lens, H, Hk, D, dtype, causal, kind, None, D + 2)


@DTYPES
@CAUSAL
@pytest.mark.parametrize("D", [32, 64, 96, 128, 192, 256])
@pytest.mark.parametrize("form", ["rows128", "keys"])
def test_split_keys(gc, form, D, causal, dtype):
    q_lens, k_lens, H, Hk, kind = SPLIT[form]
    if form == "rows128" and dtype == BF16 and D <= 128:
        k_lens = [9000, 300]     # fewer keys are not worth a split there
    run(gc, q_lens, k_lens, H, Hk, D, dtype, causal, kind, True, D + 3)


def test_eight_waves_many_rows(gc):
    """A sequence's own tokens, where the first block's rows see one tile and the last's all of them."""
    run(gc, [4095], [4095], 16, 16, 64, BF16, False, ROWS256, False, 5)
    run(gc, [256] * 16, [700] * 16, 16, 16, 128, BF16, True, ROWS256, False, 6)


MASKED = {
    "keys": ([5, 1], [300, 77], 8, 2, KEYS),
    "keys_split": ([5, 1], [300, 9000], 8, 2, KEYS),
    "rows256": ([256] * 16, [640, 641] * 8, 16, 16, ROWS256),
}


FEW_ROWS = [(32, F32), (64, F32), (80, F32), (192, F32), (64, BF16), (80, BF16), (128, BF16), (256, BF16)]


@pytest.mark.parametrize("form,D,dtype", [(form, D, dtype) for form in ("keys", "keys_split") for D, dtype in FEW_ROWS] +
                         [("rows256", D, BF16) for D in (64, 80, 128)], ids=lambda x: str(x).replace("torch.", ""))
@pytest.mark.parametrize("bad", [NAN, INF, -INF], ids=str)
def test_masked_places_have_no_effect(gc, bad, form, D, dtype):
    """Keys and values that a causal row does not see, and those of other
    sequences, hold NaN or infinity: the rows that see none of it are as
    without it, bit for bit."""
    q_lens, k_lens, H, Hk, kind = MASKED[form]
    plan = planned(gc, q_lens, k_lens, H, Hk, D, dtype, True, kind)
    q, k, v = make(q_lens, k_lens, H, Hk, D, dtype, 9)
    clean, clean_l = gc.gc_attention(q, k, v, plan)
    n, m = q_lens[0], k_lens[0]
    first = m - n + 2                 # seen by the first sequence's queries from its third on
    k2, v2 = k.clone(), v.clone()
    k2[first], v2[first, :, 5], v2[m - 1] = bad, bad, bad
    got, lse = gc.gc_attention(q, k2, v2, plan)
    rows = [i for i in range(q.shape[0]) if i < 2 or i >= n]
    assert torch.equal(got[rows], clean[rows]) and torch.equal(lse[:, rows], clean_l[:, rows])
    assert not got[2:n, :, 5].isfinite().any()
    # in values alone: the channels that see it, and no others
    got, lse = gc.gc_attention(q, k, v2, plan)
    assert torch.equal(lse, clean_l) and torch.equal(got[rows], clean[rows])
    want = torch.tensor(bad, device=DEV)
    for i in range(2, n):
        same = torch.equal(got[i, :, 5].isnan(), want.isnan().expand(H)) and (math.isnan(bad) or bool((got[i, :, 5] == bad).all()))
        assert same, i
    assert torch.equal(got[2:n - 1, :, :5], clean[2:n - 1, :, :5])
    assert not got[n - 1].isfinite().any()


@DTYPES
@pytest.mark.parametrize("q_lens,k_lens", [([3, 2], [50, 77]), ([5, 1], [300, 9000])], ids=str)
def test_padding_channels_and_next_tokens(gc, q_lens, k_lens, dtype):
    """Few rows: heads of 72 channels inside a wider buffer whose other
    channels, and the tokens after the last, hold NaN."""
    D, H = 72, 2
    plan = planned(gc, q_lens, k_lens, H, H, D, dtype, False, KEYS)
    q, k, v = make(q_lens, k_lens, H, H, D, dtype, 10)
    want = gc.gc_attention(q, k, v, plan)

    def wrap(t):
        big = torch.full((t.shape[0] + 140, H + 1, 104), NAN, dtype=dtype, device=DEV)
        big[:t.shape[0], :H, 8:8 + D] = t
        return big[:t.shape[0], :H, 8:8 + D]

    got = gc.gc_attention(wrap(q), wrap(k), wrap(v), plan, out=wrap(torch.zeros_like(q)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("D", [72, 128])
def test_padding_channels_eight_waves(gc, D):
    q_lens, k_lens, H = [256] * 16, [640, 641] * 8, 16
    plan = planned(gc, q_lens, k_lens, H, H, D, BF16, False, ROWS256)
    q, k, v = make(q_lens, k_lens, H, H, D, BF16, 11)
    want = gc.gc_attention(q, k, v, plan)

    def wrap(t):
        big = torch.full((t.shape[0] + 140, H + 1, D + 24), NAN, dtype=BF16, device=DEV)
        big[:t.shape[0], :H, 8:8 + D] = t
        return big[:t.shape[0], :H, 8:8 + D]

    got = gc.gc_attention(wrap(q), wrap(k), wrap(v), plan, out=wrap(torch.zeros_like(q)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
