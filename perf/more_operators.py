"""Workloads of the operators around a denoiser block's attention: the norm of the residual stream, rows in 8 bits, and
matrix products with what follows them.

A block of a multi-view denoiser adds its attention's output to the residual stream, norms the sum, and runs a feed-forward
part whose second product is added again.  The rows are the foreground tokens of the views at hand, or one a step
and asset where the step's time is projected.  With weights in 8 bits the norm writes its rows in 8 bits with a scale each,
and what lies between two products is laid out the same way.  The kinds (key "op"):

  norm      total = x + residual; out = total / rms(total) * gain, in the inputs' type or in 8 bits (e4m3) with a scale a row
  quantize  rows in 8 bits (e4m3) with a scale each
  linear    act(x w^T + bias) + residual, or gated act(x w^T + bias) * (x v^T + bias) + residual, with w's and v's rows one
            after the other; operands in float32, bfloat16, or 8 bits with a scale for each row of x and of w

`own` false computes the plain form in float32 with elementary torch operations; `own` true calls the library.
exact() computes the same in 64 bits.
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6
LARGEST = 448.0                      # of e4m3
SMALLEST_SCALE = 2.0 ** -126

# caps of a drawn case: values of a tensor of rows, of the weights and of the product, multiply-adds
MOST_VALUES = 196608 * 2048
MOST_WEIGHTS = 16384 * 4096
MOST_OUT = 24576 * 16384
MOST_PRODUCTS = 24576 * 4096 * 16384


def listed():
    return [
        # the time embedding of one asset between two products: launch latency
        dict(name="norm_token_bf16", op="norm", T=1, width=4096, residual=True, dtype="bf16", out="bf16", wide=0),
        # foreground tokens of two anchors, a width that is no multiple of anything, float
        dict(name="norm_odd_f32", op="norm", T=5741, width=1283, residual=True, dtype="f32", out="f32", wide=0),
        # every token of a twelve-view 128 x 128 asset, for products in 8 bits
        dict(name="norm_full_e4m3", op="norm", T=196608, width=2048, residual=True, dtype="bf16", out="e4m3", wide=0),
        # the foreground tokens of two anchors of four 48 x 48 token assets, between the feed-forward part's products
        dict(name="quant_anchors_bf16", op="quantize", T=10403, width=4096, dtype="bf16", wide=0),
        # a float weight when it is loaded: columns of a wider one
        dict(name="quant_weight_f32", op="quantize", T=16384, width=4096, dtype="f32", wide=1024),
        # one asset's time embedding, projected for all parts of a block
        dict(name="lin_token_bf16", op="linear", M=1, N=6144, K=4096, act="silu", gated=False, bias=True, residual=False,
             dtype="bf16", out="bf16", wide=0),
        # sixteen assets' embeddings, weights in 8 bits
        dict(name="lin_steps_e4m3", op="linear", M=16, N=8192, K=4096, act="gelu_tanh", gated=False, bias=True,
             residual=False, dtype="e4m3", out="bf16", wide=0),
        # one view of the 32 x 32 grid, float, an odd number of outputs
        dict(name="lin_view_f32", op="linear", M=1024, N=1283, K=1024, act="gelu", gated=False, bias=True, residual=True,
             dtype="f32", out="f32", wide=0),
        # the first product of a gated feed-forward part on the foreground tokens of two anchors of four assets
        dict(name="lin_gated_bf16", op="linear", M=10403, N=2736, K=1024, act="silu", gated=True, bias=False,
             residual=False, dtype="bf16", out="bf16", wide=0),
        # its second one, added to the residual stream; x is columns of a wider buffer
        dict(name="lin_down_bf16", op="linear", M=10403, N=1024, K=2736, act="none", gated=False, bias=True,
             residual=True, dtype="bf16", out="bf16", wide=64),
        # a wide feed-forward part on every token of a six-view 64 x 64 token asset
        dict(name="lin_full_bf16", op="linear", M=24576, N=16384, K=4096, act="gelu_tanh", gated=False, bias=True,
             residual=False, dtype="bf16", out="bf16", wide=0),
        # the same part gated, in 8 bits
        dict(name="lin_full_e4m3", op="linear", M=24576, N=8192, K=4096, act="silu", gated=True, bias=False,
             residual=False, dtype="e4m3", out="bf16", wide=0),
    ]


def _spread(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["norm", "quantize", "linear", "linear", "linear"])
    wide = rng.choice([0, 0, 64])
    if op != "linear":
        width = _spread(rng, 1, 16384)
        if rng.random() < 0.6:
            width = max(16, width // 16 * 16)
        case = dict(op=op, T=_spread(rng, 1, min(196608, MOST_VALUES // width)), width=width,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), wide=wide)
        if op == "norm":
            case["residual"] = rng.random() < 0.7
            case["out"] = rng.choice([case["dtype"], "e4m3"])
        return case
    while True:
        dtype = rng.choice(["bf16", "bf16", "e4m3", "f32"])
        M, N = _spread(rng, 1, 24576), _spread(rng, 1, 16384)
        if rng.random() < 0.6:
            N = max(16, N // 16 * 16)
        K = 16 * _spread(rng, 1, 1024) - (8 if dtype != "e4m3" and rng.random() < 0.2 else 0)
        gated = rng.random() < 0.3
        rows = 2 * N if gated else N
        # (a float product costs eight times and more)
        if rows * K > MOST_WEIGHTS or M * K > MOST_VALUES or M * rows > MOST_OUT:
            continue
        if M * rows * K * (8 if dtype == "f32" else 1) > MOST_PRODUCTS:
            continue
        return dict(op=op, M=M, N=N, K=K, act=rng.choice(["none", "silu", "gelu", "gelu_tanh"]), gated=gated,
                    bias=rng.random() < 0.6, residual=rng.random() < 0.5, dtype=dtype,
                    out="f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]), wide=wide)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rows(n, width, wide, dtype, g, size=1.0):
    """Rows with a few channels that are larger than the others; wide: columns of a buffer that has so many more."""
    x = torch.randn((n, width + wide), generator=g, device=DEV)
    x *= size * (1 + 4 * (torch.rand((width + wide,), generator=g, device=DEV) < 0.01))
    return x.to(dtype)[:, wide // 2:wide // 2 + width]


def _eight_bits(x):
    """(e4m3, scale of each row)."""
    s = x.abs().amax(-1).clamp_min(LARGEST * SMALLEST_SCALE) / LARGEST
    return (x / s[:, None]).to(torch.float8_e4m3fn), s


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1000003 + 17)
    s = dict(case)
    dtype, wide = DTYPES[case["dtype"]], case["wide"]
    if case["op"] == "linear":
        M, K, R = case["M"], case["K"], case["N"] * (2 if case["gated"] else 1)
        if case["dtype"] == "e4m3":
            x, s["x_scale"] = _eight_bits(_rows(M, K, wide, torch.float32, g))
            s["x"] = torch.empty((M, K + wide), dtype=dtype, device=DEV)[:, wide // 2:wide // 2 + K]
            s["x"].copy_(x)
            s["w"], s["w_scale"] = _eight_bits(torch.randn((R, K), generator=g, device=DEV) / math.sqrt(K))
        else:
            s["x"] = _rows(M, K, wide, dtype, g)
            s["w"] = (torch.randn((R, K), generator=g, device=DEV) / math.sqrt(K)).to(dtype)
            s["x_scale"] = s["w_scale"] = None
        s["b"] = torch.randn((R,), generator=g, device=DEV) * 0.1 if case["bias"] else None
        s["r"] = _rows(M, case["N"], 0, DTYPES[case["out"]], g) if case["residual"] else None
    else:
        s["x"] = _rows(case["T"], case["width"], wide, dtype, g)
        if case["op"] == "norm":
            s["r"] = _rows(case["T"], case["width"], 0, dtype, g, 3.0) if case["residual"] else None
            s["gain"] = 1 + 0.2 * torch.randn((case["width"],), generator=g, device=DEV)
    if own:
        import paper_2608_13255_amd as gc
        s["gc"] = gc
        s["code"] = {"none": gc.GC_ACT_NONE, "silu": gc.GC_ACT_SILU, "gelu": gc.GC_ACT_GELU,
                     "gelu_tanh": gc.GC_ACT_GELU_TANH}[case.get("act", "none")]
    return s


# ---------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------

def _act(x, kind):
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _plain_linear(s):
    p = s["x"].float() @ s["w"].float().t()
    if s["x_scale"] is not None:
        p = p * s["x_scale"][:, None] * s["w_scale"]
    if s["b"] is not None:
        p = p + s["b"]
    p = _act(p[:, :s["N"]], s["act"]) * p[:, s["N"]:] if s["gated"] else _act(p, s["act"])
    if s["r"] is not None:
        p = p + s["r"].float()
    return p.to(DTYPES[s["out"]])


def run(s):
    if s["op"] == "linear":
        if own:
            return s["gc"].gc_linear(s["x"], s["w"], bias=s["b"], act=s["code"], gated=s["gated"], residual=s["r"],
                                     x_scale=s["x_scale"], w_scale=s["w_scale"], out_dtype=DTYPES[s["out"]])
        return _plain_linear(s)
    if s["op"] == "quantize":
        if own:
            return s["gc"].gc_quantize_rows(s["x"])
        return _eight_bits(s["x"].float())
    if own:
        out, scale, total = s["gc"].gc_add_rms_norm(s["x"], residual=s["r"], gain=s["gain"], eps=EPS,
                                                    out_dtype=DTYPES[s["out"]])
    else:
        h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["gain"]
        out, scale = _eight_bits(y) if s["out"] == "e4m3" else (y.to(s["x"].dtype), None)
        total = h.to(s["x"].dtype)
    return out, scale, None if s["r"] is None else total


def work(case):
    size = {"f32": 4, "bf16": 2, "e4m3": 1}
    e = size[case["dtype"]]
    if case["op"] == "linear":
        M, N, K, R = case["M"], case["N"], case["K"], case["N"] * (2 if case["gated"] else 1)
        b = (M + R) * K * e + M * N * size[case["out"]] * (2 if case["residual"] else 1)
        b += 4 * R * (1 if case["bias"] else 0) + (4 * (M + R) if case["dtype"] == "e4m3" else 0)
        return {"bytes": b, "flops": 2 * M * R * K}
    n = case["T"] * case["width"]
    if case["op"] == "quantize":
        return {"bytes": n * (e + 1) + 4 * case["T"], "flops": 2 * n}
    b = n * (e + size[case["out"]] + (2 * e if case["residual"] else 0)) + 4 * case["width"]
    return {"bytes": b + (4 * case["T"] if case["out"] == "e4m3" else 0), "flops": 5 * n}


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------

def _exact_act(x, kind):
    if kind == "silu":
        return x * torch.sigmoid(x)
    if kind == "gelu":
        return x * torch.special.erfc(x / -2 ** 0.5) / 2
    if kind == "gelu_tanh":     # (1 + tanh u) / 2 is the logistic function of 2 u
        return x * torch.sigmoid((8 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3))
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "linear":
        M, N = s["M"], s["N"]
        w = s["w"].double()
        if s["w_scale"] is not None:
            w = w * s["w_scale"].double()[:, None]
        out = torch.empty((M, N), dtype=torch.float64, device=DEV)
        for i in range(0, M, 4096):
            x = s["x"][i:i + 4096].double()
            if s["x_scale"] is not None:
                x = x * s["x_scale"][i:i + 4096].double()[:, None]
            p = torch.nn.functional.linear(x, w)
            if s["b"] is not None:
                p = p + s["b"].double()
            y = _exact_act(p[:, :N], s["act"])
            if s["gated"]:
                y = y * p[:, N:]
            out[i:i + 4096] = y if s["r"] is None else y + s["r"][i:i + 4096].double()
        return out
    x = s["x"].double()
    if s["op"] == "norm":
        if s["r"] is not None:
            x += s["r"].double()
        total = None if s["r"] is None else x.clone()
        x *= (s["gain"].double() / (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / s["width"] + EPS).sqrt())
        if s["out"] != "e4m3":
            return x, None, total
    scale = torch.linalg.vector_norm(x, ord=math.inf, dim=-1).clamp(min=LARGEST * SMALLEST_SCALE) / LARGEST
    x /= scale[:, None]
    return (x, scale, total) if s["op"] == "norm" else (x, scale)
