"""Calls on an explicit stream that the current stream is not ordered with:
their outputs and workspaces lie in no memory that current-stream work may
still use, and stay their own while either stream uses them."""
import pytest
import torch

import synth
from synth.configs import C2

from conftest import latent_maps

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SLEEP = 40_000_000


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


def randn(shape, seed, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def stream_beside():
    """A stream whose work does not wait for the current one's (streams may share a hardware queue)."""
    probe = torch.zeros(1, device=DEV)
    for _ in range(8):
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        torch.cuda._sleep(SLEEP)
        with torch.cuda.stream(s):
            probe.add_(1)
        s.synchronize()
        held = not torch.cuda.current_stream().query()
        torch.cuda.synchronize()
        if held:
            return s
    pytest.skip("every stream shares the current one's queue")


def calls(gc):
    w = C2
    P = torch.from_numpy(latent_maps(w.name, 1)).to(DEV)
    N, H, W = P.shape[1:4]
    cams = gc.camera_tensor({k: v[:1] for k, v in synth.batch_cameras(w).items()}, DEV)
    bbox = gc.gc_posmap_bbox(P)
    A = gc.gc_schedule_anchors(N, w.a, 0)
    corr, wts = gc.gc_build_correspondence(P, cams, A, w.K, bbox)
    pairs, stale = gc.gc_coverage_pairs(P, cams, bbox), gc.gc_coverage_init(P)
    x0, xt = randn((1, N, H, W, 8), 1), randn((1, N, H, W, 8), 2)
    new = randn((1, w.a, H, W, 8), 3)
    smp = gc.Sampler(kind=gc.GC_FLOW_EULER, pred_out=gc.GC_PRED_VEL)
    st = gc.gc_unipc_coeffs(gc.Sampler(kind=gc.GC_DDIM), 10, 0, 1, False)
    x, r = randn((900, 320), 4), randn((900, 320), 5)
    a, b = randn((120, 8192), 6), randn((256, 8192), 7)
    assert gc.gc_linear_workspace_bytes(120, 256, 8192, torch.bfloat16) > 0
    q, k, v = (randn((3000, h, 64), 8 + h) for h in (4, 2, 2))
    plan = gc.gc_attention_plan([3000], [3000], 4, 2, 64, torch.bfloat16, device=DEV)
    assert plan.info.workspace_bytes > 0
    table = gc.gc_rope_table(3000, [32], device=DEV)
    at = torch.arange(3000, dtype=torch.int32, device=DEV)
    gain = torch.ones(64, device=DEV)
    return {
        "linear": lambda s: gc.gc_linear(a, b, stream=s),
        "norm": lambda s: gc.gc_add_rms_norm(x, residual=r, out_dtype=torch.float8_e4m3fn, stream=s),
        "quantize": lambda s: gc.gc_quantize_rows(x, stream=s),
        "attention": lambda s: gc.gc_attention(q, k, v, plan, stream=s),
        "rope": lambda s: gc.gc_rope(q, at, table, stream=s),
        "qk_norm_rope": lambda s: gc.gc_qk_norm_rope(q, k, gain, gain, at, table, stream=s),
        "rope_table": lambda s: gc.gc_rope_table(3000, [32], device=DEV, stream=s),
        "bbox": lambda s: gc.gc_posmap_bbox(P, stream=s),
        "correspondence": lambda s: gc.gc_build_correspondence(P, cams, A, w.K, bbox, stream=s)[0],
        "index": lambda s: gc.gc_index_correspondence(corr, stream=s).vis_bits,
        "index_foreground": lambda s: gc.gc_index_foreground(P, stream=s).fg_bits,
        "transport": lambda s: gc.gc_transport_step(x0, new, corr, wts, A, stream=s),
        "reconstruct": lambda s: gc.gc_transport_reconstruct(x0, new, corr, wts, xt, A, smp, 0.8, 0.6, stream=s),
        "geom": lambda s: gc.gc_transport_reconstruct_geom(x0, new, P, cams, bbox, xt, A, w.K, smp, 0.8, 0.6, stream=s),
        "sampler": lambda s: gc.gc_sampler_reconstruct(xt, x0, smp, 0.8, 0.6, stream=s),
        "unipc": lambda s: gc.gc_transport_unipc(x0, new, corr, wts, A, st, x_cur=xt, stream=s),
        "pairs": lambda s: gc.gc_coverage_pairs(P, cams, bbox, stream=s),
        "coverage_init": lambda s: gc.gc_coverage_init(P, stream=s),
        "select": lambda s: gc.gc_coverage_select(pairs, stale, w.a, stream=s),
        "score": lambda s: gc.gc_coverage_score(pairs, stale, [A], stream=s),
    }


NAMES = ["linear", "norm", "quantize", "attention", "rope", "qk_norm_rope", "rope_table", "bbox", "correspondence", "index",
         "index_foreground", "transport", "reconstruct", "geom", "sampler", "unipc", "pairs", "coverage_init", "select", "score"]


def tensors(got):
    return [t for t in (got if isinstance(got, tuple) else (got,)) if t is not None]


def raw(t):
    return t.contiguous().view(torch.uint8)


@pytest.fixture(scope="module")
def table(gc):
    return calls(gc)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("handle", [False, True])
def test_outputs_and_workspaces(gc, monkeypatch, table, name, handle):
    """What a call on the current stream gave back lies free for that stream, whose work with it has yet to end: a call of the
    same sizes on another stream takes other memory for all that it allocates."""
    call = table[name]
    want = [t.clone() for t in tensors(call(None))]
    s = stream_beside()
    taken = []
    real = torch.empty

    def empty(*args, **kwargs):
        taken.append(real(*args, **kwargs))
        return taken[-1]

    def empty_like(*args, **kwargs):
        taken.append(real_like(*args, **kwargs))
        return taken[-1]

    real_like = torch.empty_like
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", empty)
        m.setattr(torch, "empty_like", empty_like)
        first = call(None) if not name.startswith("index") else None     # (those read back: they would wait for the current stream)
        used = {t.data_ptr() for t in taken + ([] if first is None else tensors(first))}
        del first
        taken.clear()
        got = call(s.cuda_stream if handle else s)
    after = {t.data_ptr() for t in taken}
    assert after and not (used & after)
    assert name.startswith("index") or not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    for a, b in zip(tensors(got), want):
        assert torch.equal(raw(a), raw(b))


def test_parts_of_two_calls_stay_apart(gc):
    """Two products whose inner dimension is cut, on the current stream and another, nothing between them."""
    s = stream_beside()
    jobs = [(randn((120, 8192), 30 + i), randn((256, 8192), 40 + i)) for i in range(2)]
    want = [gc.gc_linear(*j) for j in jobs]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [gc.gc_linear(*jobs[0]), gc.gc_linear(*jobs[1], stream=s)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_an_output_dropped_while_the_current_stream_reads_it(gc):
    """A side stream's output that the current stream has yet to read is not handed to the side stream's next work."""
    x = randn((900, 320), 50)
    s = stream_beside()
    with torch.cuda.stream(s):
        want = gc.gc_add_rms_norm(x)[0].clone()
    torch.cuda.synchronize()
    out = gc.gc_add_rms_norm(x, stream=s)[0]
    s.synchronize()
    torch.cuda._sleep(SLEEP)
    read = out.clone()
    at = out.data_ptr()
    del out
    with torch.cuda.stream(s):
        later = [torch.full((900, 320), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    held = not torch.cuda.current_stream().query()
    assert held and at not in {t.data_ptr() for t in later}
    torch.cuda.synchronize()
    assert torch.equal(read, want)
