"""What the norms and matrix products of the denoiser's blocks refuse on the host, before any launch (no GPU)."""
import ctypes
import math

import pytest
import torch

# never-dereferenced device addresses: every call with them fails validation
A = [0x100000000 * (i + 1) for i in range(12)]
CODE = {v: k for k, v in {-1: "ARG", -2: "SHAPE", -3: "DTYPE", -4: "ALIGN", -5: "ALIAS", -6: "CAPACITY"}.items()}
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


@pytest.fixture(scope="module")
def L(gc):
    return gc.lib()


def refused(L, rc, code, *words):
    text = L.gc_last_error().decode()
    assert rc == CODE[code], (rc, text)
    for w in words:
        assert w in text, text


def ref(gc, data, stride):
    return None if data is None else ctypes.byref(gc._Rows(data, stride))


def test_struct_size_and_codes(gc):
    assert ctypes.sizeof(gc._Rows) == 16
    assert (gc.GC_F32, gc.GC_BF16, gc.GC_E4M3) == (F32, BF16, E4M3)


def norm(gc, L, x=(A[0], 64), r=None, n=10, width=64, dtype=BF16, gain=A[5], eps=1e-6, total=None, out=(A[1], 64), out_dtype=BF16,
         scale=None):
    return L.gc_add_rms_norm(ref(gc, *x), ref(gc, *r) if r else None, n, width, dtype, gain, eps,
                             ref(gc, *total) if total else None, ref(gc, *out), out_dtype, scale, None)


def test_norm_refusals(gc, L):
    refused(L, norm(gc, L, dtype=7), "DTYPE")
    refused(L, norm(gc, L, dtype=E4M3, out_dtype=E4M3), "DTYPE")
    refused(L, norm(gc, L, out_dtype=F32), "DTYPE", "out_dtype")
    refused(L, norm(gc, L, n=-1), "CAPACITY", "n_rows")
    refused(L, norm(gc, L, n=2 ** 31), "CAPACITY", "n_rows")
    refused(L, norm(gc, L, width=0), "CAPACITY", "width")
    refused(L, norm(gc, L, width=32769), "CAPACITY", "width")
    for eps in (-1e-6, math.nan, math.inf, 1e-60, 7e-46, 3.5e38):
        refused(L, norm(gc, L, eps=eps), "ARG", "eps")
    refused(L, norm(gc, L, x=(None, 0)), "ARG", "x is null")
    refused(L, norm(gc, L, out=(None, 0)), "ARG", "out is null")
    refused(L, norm(gc, L, x=(A[0] + 1, 64)), "ALIGN", "x")
    refused(L, norm(gc, L, r=(A[2] + 1, 64)), "ALIGN", "residual")
    refused(L, norm(gc, L, gain=A[5] + 2), "ALIGN", "gain")
    refused(L, norm(gc, L, x=(A[0], -64)), "SHAPE", "stride")
    refused(L, norm(gc, L, out=(A[1], 63)), "SHAPE", "rows overlap")
    refused(L, norm(gc, L, total=(A[1] + 0x1000000, 0)), "SHAPE", "total")
    refused(L, norm(gc, L, scale=A[6]), "ARG", "8-bit")
    refused(L, norm(gc, L, out_dtype=E4M3), "ARG", "out_scale")
    refused(L, norm(gc, L, out_dtype=E4M3, scale=A[6] + 2), "ALIGN", "out_scale")
    refused(L, norm(gc, L, out=(A[0] + 64, 64)), "ALIAS", "out overlaps x")
    refused(L, norm(gc, L, out=(A[0], 64), out_dtype=E4M3, scale=A[6]), "ALIAS", "out overlaps x")     # 8 bits where 16 lie
    refused(L, norm(gc, L, out=(A[0], 65)), "ALIAS", "out overlaps x")                                 # its place, another stride
    refused(L, norm(gc, L, r=(A[2], 64), total=(A[2] + 2, 64)), "ALIAS", "total overlaps residual")
    refused(L, norm(gc, L, total=(A[1], 64)), "ALIAS", "total overlaps out")
    refused(L, norm(gc, L, out=(A[5], 64)), "ALIAS", "gain")
    refused(L, norm(gc, L, out_dtype=E4M3, scale=A[0]), "ALIAS", "out_scale overlaps x")
    refused(L, norm(gc, L, out_dtype=E4M3, scale=A[1] + 8), "ALIAS", "out")
    # up to the gain's check (misaligned here) these are taken: in place, and columns of one buffer
    for more in (dict(out=(A[0], 64)), dict(r=(A[2], 64), total=(A[2], 64)), dict(x=(A[0], 256), out=(A[0] + 128, 256)),
                 dict(x=(A[0], 0)), dict(total=(A[0], 64))):
        more.setdefault("gain", A[5] + 2)
        refused(L, norm(gc, L, **more), "ALIGN", "gain")
    assert norm(gc, L, n=0, x=(None, 0), out=(None, 0)) == 0


def test_quantize_refusals(gc, L):
    def call(x=(A[0], 64), n=10, width=64, dtype=BF16, out=(A[1], 64), scale=A[2]):
        return L.gc_quantize_rows(ref(gc, *x), n, width, dtype, ref(gc, *out), scale, None)
    refused(L, call(dtype=E4M3), "DTYPE")
    refused(L, call(width=-3), "CAPACITY")
    refused(L, call(n=-2), "CAPACITY")
    refused(L, call(x=(None, 0)), "ARG", "x")
    refused(L, call(scale=None), "ARG", "out_scale")
    refused(L, call(out=(A[1], 12)), "SHAPE", "out")
    refused(L, call(out=(A[0] + 8, 64)), "ALIAS")
    refused(L, call(scale=A[0] + 4), "ALIAS", "x")
    refused(L, call(scale=A[1] + 4), "ALIAS", "out")
    assert call(n=0, x=(None, 0), out=(None, 0), scale=None) == 0


def linear(gc, L, x=(A[0], 64), xs=None, w=(A[1], 64), ws=None, n=10, n_out=48, n_in=64, dtype=BF16, bias=None, act=0, gated=0,
           r=None, out=(A[2], 48), out_dtype=BF16, work=A[3], size=1 << 40):
    return L.gc_linear(ref(gc, *x), xs, ref(gc, *w), ws, n, n_out, n_in, dtype, bias, act, gated, ref(gc, *r) if r else None,
                       ref(gc, *out), out_dtype, work, size, None)


def test_linear_refusals(gc, L):
    refused(L, linear(gc, L, dtype=3), "DTYPE")
    refused(L, linear(gc, L, dtype=F32, x=(A[0], 64), w=(A[1], 64)), "DTYPE", "out_dtype")      # bfloat16 of float32
    refused(L, linear(gc, L, out_dtype=E4M3), "DTYPE", "out_dtype")
    refused(L, linear(gc, L, n=-1), "CAPACITY", "n_rows")
    refused(L, linear(gc, L, n_out=0), "CAPACITY", "n_out")
    refused(L, linear(gc, L, n_out=(1 << 22) + 1), "CAPACITY", "n_out")
    refused(L, linear(gc, L, n_in=0), "CAPACITY", "n_in")
    refused(L, linear(gc, L, n_in=(1 << 20) + 8), "CAPACITY", "n_in")
    refused(L, linear(gc, L, n_in=60), "SHAPE", "n_in")
    refused(L, linear(gc, L, n_in=56, dtype=E4M3), "SHAPE", "n_in")
    for act in (-1, 4):
        refused(L, linear(gc, L, act=act), "ARG", "activation")
    refused(L, linear(gc, L, xs=A[4]), "ARG", "scales")
    refused(L, linear(gc, L, ws=A[4]), "ARG", "scales")
    refused(L, linear(gc, L, x=(None, 0)), "ARG", "x is null")
    refused(L, linear(gc, L, w=(None, 0)), "ARG", "w is null")
    refused(L, linear(gc, L, out=(None, 0)), "ARG", "out is null")
    refused(L, linear(gc, L, x=(A[0] + 8, 64)), "ALIGN", "x")
    refused(L, linear(gc, L, w=(A[1], 68)), "ALIGN", "w")
    refused(L, linear(gc, L, x=(A[0], (1 << 20) + 8)), "SHAPE", "x")
    refused(L, linear(gc, L, w=(A[1], -64)), "SHAPE", "w")
    refused(L, linear(gc, L, out=(A[2], 40)), "SHAPE", "out")
    refused(L, linear(gc, L, out=(A[2] + 1, 48)), "ALIGN", "out")
    refused(L, linear(gc, L, bias=A[4] + 2), "ALIGN", "bias")
    refused(L, linear(gc, L, r=(A[4] + 1, 48)), "ALIGN", "residual")
    refused(L, linear(gc, L, out=(A[0], 48)), "ALIAS", "out overlaps x")
    refused(L, linear(gc, L, out=(A[1], 48)), "ALIAS", "out overlaps w")
    refused(L, linear(gc, L, gated=1, out=(A[1] + 48 * 128, 48)), "ALIAS", "out overlaps w")     # the values' rows
    refused(L, linear(gc, L, r=(A[2] + 2, 48)), "ALIAS", "residual")
    refused(L, linear(gc, L, r=(A[2], 56)), "ALIAS", "residual")
    refused(L, linear(gc, L, bias=A[2] + 8), "ALIAS", "bias")
    refused(L, linear(gc, L, dtype=E4M3, xs=A[2]), "ALIAS", "x_scale")
    assert linear(gc, L, n=0, x=(None, 0), w=(None, 0), out=(None, 0), work=None, size=0) == 0


@pytest.mark.parametrize("gated", [0, 1])
def test_linear_workspace(gc, L, gated):
    """A long inner dimension and few tiles: parts, whose sums pass through the workspace."""
    sizes = dict(n=100, n_out=64, n_in=8192, x=(A[0], 8192), w=(A[1], 8192), out=(A[2], 64), gated=gated)
    need = L.gc_linear_workspace_bytes(100, 64, 8192, BF16, gated)
    assert need > 0 and need % (100 * 64 * 4 * (1 + gated)) == 0
    refused(L, linear(gc, L, work=None, **sizes), "ARG", "workspace")
    refused(L, linear(gc, L, size=need - 1, **sizes), "CAPACITY", "workspace")
    refused(L, linear(gc, L, work=A[3] + 8, **sizes), "ALIGN", "workspace")
    for other in (A[0], A[1], A[2]):
        refused(L, linear(gc, L, work=other, **sizes), "ALIAS", "workspace")
    refused(L, linear(gc, L, r=(A[4], 64), work=A[4] + 16, **sizes), "ALIAS", "workspace")
    refused(L, linear(gc, L, bias=A[4], work=A[4], **sizes), "ALIAS", "workspace")
    assert L.gc_linear_workspace_bytes(10000, 4096, 64, BF16, gated) == 0
    for bad in ((-1, 64, 64, BF16), (1, 0, 64, BF16), (1, 64, 60, BF16), (1, 64, 64, 5)):
        assert L.gc_linear_workspace_bytes(*bad, gated) == -1


def test_workspace_holds_for_every_size(gc, L):
    """Whole parts of whole rows, never more than 16 of them, and none where they would not be read."""
    for dtype, unit in ((F32, 4), (BF16, 8), (E4M3, 16)):
        for n in (1, 16, 17, 64, 100, 513, 4096, 100000):
            for n_out in (1, 7, 64, 1000, 16384):
                for n_in in (unit, 40 * unit, 1000 * unit):
                    for gated in (0, 1):
                        need = L.gc_linear_workspace_bytes(n, n_out, n_in, dtype, gated)
                        part = n * ((n_out + 7) // 8 * 8) * 4 * (1 + gated)
                        assert need == 0 or (need % part == 0 and 2 <= need // part <= 16)


def test_binding_refusals(gc):
    x, w = torch.zeros((4, 32)), torch.zeros((6, 32))
    with pytest.raises(ValueError, match="device tensor"):
        gc.gc_linear(x, w)
    with pytest.raises(ValueError, match="device tensor"):
        gc.gc_add_rms_norm(x)
    with pytest.raises(ValueError, match="device tensor"):
        gc.gc_quantize_rows(x)
    with pytest.raises(TypeError):
        gc.gc_linear([1.0], w)
    with pytest.raises(gc.GeoCacheError):
        gc.gc_linear_workspace_bytes(4, 6, 33, torch.bfloat16)
    with pytest.raises(gc.GeoCacheError):
        gc.gc_linear_workspace_bytes(4, 6, 32, torch.float16)
    for sizes in ((4, 2 ** 32 + 6, 32), (4, 6, 2 ** 32 + 32), (2 ** 31, 6, 32), (4, -1, 32)):
        with pytest.raises(ValueError, match="2\\^31"):
            gc.gc_linear_workspace_bytes(*sizes, torch.bfloat16)
