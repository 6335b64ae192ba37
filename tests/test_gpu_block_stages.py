"""Each stage of MultiViewBlock against the same in 64 bits, element by element, on what the stage before really gave it: a
gain, bias, weight, scale or residual that is left out, or another's, shows in its own stage, whatever the stages after make of
it.

The operators are replaced by ones that also keep a copy of what they return; what a stage should have returned follows from
the copies before it and the block's own tensors alone.  With u = 2^-24 and half a step of the stored type t, h = eps(t) / 2:
  norms        a mean of squares of at most 256 columns: lanes of at most 8 squares and a tree, under 24 u, half of that after
               the root; the products with it and the gain add a few: 20 u |y| and h |y|
  products     (K + 8) u of the magnitudes' sum, the epilogue's 20 u, h |y|; 8-bit operands with a bfloat16 result: 2^-7 of the
               largest product of each 64 columns beside that
  8-bit rows   a scale off by as much as its row's values and 2 u, values by half a step, 2^-4 of themselves or 2^-10 scales
  rotation     the norm's 20 u and 8 u of |a| + |b| for two products, cosine and sine; h |y|
  attention    scores are sums of 64 products, off by 68 u of the magnitudes' sum, which is at most sqrt(64) 1.61^2 = 20.8 (gains
               are below 1.61): by 8.5e-5; a weight by twice that, and by the exponential's and the sums' own 4e-5 (of fewer
               than 400 keys): below 2^-12; weights are rounded to the type for the products, h of each: (2^-12 + h) sum p |v|
               and h |y|"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
E4M3 = torch.float8_e4m3fn
WIDTH, HEADS, KV, DIM, HIDDEN = 64, 4, 2, 64, 176
VIEWS = [4, 1]


class Recorder:
    """The operators of a block, with copies of what they return."""

    def __init__(self, monkeypatch):
        from paper_2608_13255_amd import multiview
        self.got = []
        for name in ("gc_add_rms_norm", "gc_linear", "gc_quantize_rows", "gc_attention", "gc_qk_norm_rope"):
            monkeypatch.setattr(multiview, name, self.wrapped(getattr(multiview, name), name))

    def wrapped(self, real, name):
        def call(*args, **kwargs):
            out = real(*args, **kwargs)
            self.got.append((name, [None if t is None else t.clone() for t in (out if isinstance(out, tuple) else (out,))]))
            return out
        return call

    def next(self, name):
        at, out = self.got.pop(0)
        assert at == name, (at, name)
        return out


def block_for(dtype, gated, act, biases):
    from paper_2608_13255_amd.multiview import MultiViewBlock
    g = torch.Generator(device=DEV)
    g.manual_seed(31)
    pos = torch.randn((2, 6, 12, 16, 3), generator=g, device=DEV)
    pos[torch.rand(pos.shape[:4], generator=g, device=DEV) < 0.4] = math.nan
    block = MultiViewBlock(pos, WIDTH, HEADS, KV, DIM, HIDDEN, act=act, gated=gated, dtype=dtype, generator=g)
    for gain in (block.q_gain, block.k_gain, block.attention_gain, block.feed_gain):
        gain.copy_(1 + 0.3 * torch.randn(gain.shape, generator=g, device=DEV).clamp(-2, 2))
    if biases:
        for name in ("qkv", "out", "in", "down"):
            setattr(block, "b_" + name, 0.3 * torch.randn(getattr(block, "w_" + name).shape[0], generator=g, device=DEV))
    return block, g


def near(got, want, err, label):
    half = torch.finfo(got.dtype).eps / 2
    bad = (got.double() - want).abs() - err - half * (want.abs() + err) - torch.finfo(got.dtype).tiny
    assert torch.isfinite(got).all(), label
    assert float(bad.max()) <= 0, (label, float(bad.max()))


def near_eight(q, scale, want, err, label):
    """8-bit rows with scales; err: how far the values may be off before they are rounded."""
    top = want.abs().amax(-1).clamp_min(448 * 2.0 ** -126)
    off = err.amax(-1) if torch.is_tensor(err) else torch.zeros_like(top)
    assert float(((scale.double() * 448 - top).abs() - off - 3 * U * top).max()) <= 0, label
    s = scale.double()[:, None]
    bad = (q.double() * s - want).abs() - err - 2.0 ** -4 * (1 + 8 * U) * (want.abs() + err) - 2.0 ** -10 * s
    assert float(bad.max()) <= 0, (label, float(bad.max()))


def norm64(u, gain, eps=1e-6):
    return u / (u.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()


def act64(p, act):
    return {0: p, 1: p * torch.sigmoid(p), 2: p * torch.special.erfc(-p / math.sqrt(2)) / 2}[act]


class Product:
    """A stage's product in 64 bits, and how far float32 (or the 8-bit units) may be off."""

    def __init__(self, block, name, x, eight):
        w = getattr(block, "w_" + name).double()
        if eight:
            scale = w.abs().amax(-1, keepdim=True) / 448
            q = block.eight_bits["w_" + name]
            near_eight(*q, w, 0.0 * w, "w_" + name)
            w = q[0].double() * q[1].double()[:, None]
            assert float((q[1].double() / scale[:, 0] - 1).abs().max()) <= 3 * U
        bias = getattr(block, "b_" + name)
        self.p = x @ w.t() + (0 if bias is None else bias.double())
        self.off = (x.shape[1] + 8) * U * (x.abs() @ w.abs().t() + self.p.abs())
        if eight and block.dtype == torch.bfloat16:
            for k in range(0, x.shape[1], 64):
                self.off += 2.0 ** -7 * (x[:, None, k:k + 64].abs() * w[None, :, k:k + 64].abs()).amax(-1)

    def plain(self):
        return self.p, self.off + 20 * U * self.p.abs()

    def activated(self, act, gated):
        n = self.p.shape[1] // 2 if gated else self.p.shape[1]
        p, off = self.p[:, :n], self.off[:, :n]
        y, err = act64(p, act), 1.13 * off + 20 * U * p.abs().clamp_min(1.0)
        if not gated:
            return y, err
        v, v_off = self.p[:, n:], self.off[:, n:]
        return y * v, err * (v.abs() + v_off) + v_off * y.abs() + 4 * U * (y * v).abs()


def check_stages(block, x, y, seen, eight):
    half = torch.finfo(block.dtype).eps / 2

    def rows_of(t, err, label):
        """The operand of a product: what the block's quantization made of t, checked, or t itself."""
        if not eight:
            return t
        q, scale = seen.next("gc_quantize_rows")
        near_eight(q, scale, t, err, label)
        return q.double() * scale.double()[:, None]

    def normed(want, label):
        n, scale, total = seen.next("gc_add_rms_norm")
        if not eight:
            assert scale is None
            near(n, want, 20 * U * want.abs(), label)
            return n.double(), total
        assert n.dtype == E4M3
        near_eight(n, scale, want, 20 * U * want.abs(), label)
        return n.double() * scale.double()[:, None], total

    fg = block.foreground[:, VIEWS]
    tokens = x[fg].double()                                       # asset by asset, view by view, row by row
    n, _ = normed(norm64(tokens, block.attention_gain), "first norm")

    qkv, = seen.next("gc_linear")
    near(qkv, *Product(block, "qkv", n, eight).plain(), "qkv")
    heads = qkv.double().view(-1, HEADS + 2 * KV, DIM)

    at = fg.nonzero()
    place = torch.stack([torch.tensor(VIEWS, device=DEV)[at[:, 1]], at[:, 2], at[:, 3]], 1).double()
    freq = torch.cat([10000.0 ** (-torch.arange(m, dtype=torch.float64, device=DEV) / m) for m in block.sections])
    axis = torch.cat([torch.full((m,), a, device=DEV) for a, m in enumerate(block.sections)])
    angle = (place[:, axis] * freq)[:, None]
    c, s = angle.cos(), angle.sin()
    q, k = seen.next("gc_qk_norm_rope")
    for turned, first, count, gain, label in ((q, 0, HEADS, block.q_gain, "queries"), (k, HEADS, KV, block.k_gain, "keys")):
        u = norm64(heads[:, first:first + count], gain)
        a, b = u[..., :DIM // 2], u[..., DIM // 2:]
        want = torch.cat([a * c - b * s, b * c + a * s], -1)
        near(turned, want, 28 * U * torch.cat([a.abs() + b.abs()] * 2, -1), label)

    o, _ = seen.next("gc_attention")
    v = heads[:, HEADS + KV:]
    assert int(fg.flatten(1).sum(1).max()) < 400 and max(float(t.max()) for t in (block.q_gain, block.k_gain)) < 1.61
    asset = at[:, 0]
    other = asset[:, None] != asset[None, :]
    for i in range(HEADS):
        j = i * KV // HEADS
        scores = (q[:, i].double() @ k[:, j].double().t() / math.sqrt(DIM)).masked_fill(other, -math.inf)
        p = torch.softmax(scores, -1)
        near(o[:, i], p @ v[:, j], (2.0 ** -12 + half) * (p @ v[:, j].abs()), f"attention, head {i}")

    o = o.double().view(-1, HEADS * DIM)
    operand = rows_of(o, 0.0 * o, "attention's output")
    out, = seen.next("gc_linear")
    near(out, *Product(block, "out", operand, eight).plain(), "out")

    h = out.double() + tokens
    n, total = normed(norm64(h, block.feed_gain), "second norm")
    near(total, h, U * h.abs(), "residual stream")

    m, = seen.next("gc_linear")
    near(m, *Product(block, "in", n, eight).activated(block.act, block.gated), "in")
    m = m.double()
    operand = rows_of(m, 0.0 * m, "middle")
    last, = seen.next("gc_linear")
    p, err = Product(block, "down", operand, eight).plain()
    near(last, p + total.double(), err + 2 * U * (p.abs() + total.double().abs()), "down")

    assert not seen.got
    assert torch.equal(y[fg], last) and bool((y[~fg] == 0).all())


def called(monkeypatch, dtype, gated, act, biases, eight):
    block, g = block_for(dtype, gated, act, biases)
    if eight:
        block.lay_out_in_8_bits()
    x = torch.randn((2, len(VIEWS), 12, 16, WIDTH), generator=g, device=DEV).to(dtype)
    seen = Recorder(monkeypatch)
    return block, x, block(x, VIEWS), seen, eight


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gated,act,biases", [(True, 1, True), (False, 2, False), (True, 2, True), (False, 1, True)])
@pytest.mark.parametrize("eight", [False, True], ids=["own", "8bits"])
def test_stages(monkeypatch, dtype, gated, act, biases, eight):
    check_stages(*called(monkeypatch, dtype, gated, act, biases, eight))


@pytest.mark.parametrize("name", ["attention_gain", "feed_gain", "q_gain", "k_gain", "b_qkv", "b_out", "b_in", "b_down"])
@pytest.mark.parametrize("eight", [False, True], ids=["own", "8bits"])
def test_a_part_left_out_shows(monkeypatch, name, eight):
    """The 64-bit form without one of the block's gains or biases is not what the block computes, by these bounds."""
    block, *rest = called(monkeypatch, torch.bfloat16, True, 1, True, eight)
    getattr(block, name).fill_(1.0 if name.endswith("gain") else 0.0)
    with pytest.raises(AssertionError):
        check_stages(block, *rest)
