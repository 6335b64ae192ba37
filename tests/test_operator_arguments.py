"""What the denoiser-side operators refuse on the host, before any launch, and
the attention plan's items (no GPU)."""
import ctypes
import math
import subprocess
import sys
from pathlib import Path

import numpy as np
import pytest
import torch

# never-dereferenced device addresses: every call with them fails validation
A = [0x100000000 * (i + 1) for i in range(12)]
CODE = {v: k for k, v in {-1: "ARG", -2: "SHAPE", -3: "DTYPE", -4: "ALIGN", -5: "ALIAS", -6: "CAPACITY"}.items()}


@pytest.fixture(scope="module")
def gc():
    import paper_2608_13255_amd as gc
    return gc


@pytest.fixture(scope="module")
def L(gc):
    return gc.lib()


def heads(gc, data, token=None, head=64, n=4, dim=64):
    return gc._Heads(data, n * dim if token is None else token, head)


def i32(*v):
    return (ctypes.c_int32 * len(v))(*v)


def refused(L, rc, code, *words):
    text = L.gc_last_error().decode()
    assert rc == CODE[code], (rc, text)
    for w in words:
        assert w in text, text


def test_struct_sizes(gc):
    assert ctypes.sizeof(gc._Heads) == 24
    assert ctypes.sizeof(gc.RopeScaling) == 40
    assert ctypes.sizeof(gc.AttentionInfo) == 72


def test_table_refusals(gc, L):
    def call(table=A[0], n_pos=10, sec=(4, 4), base=1e4, scaling=None):
        return L.gc_rope_table(table, n_pos, i32(*sec) if sec is not None else None, len(sec or ()), base,
                               ctypes.byref(scaling) if scaling else None, None)
    refused(L, call(table=None), "ARG", "table")
    refused(L, call(table=A[0] + 4), "ALIGN")
    refused(L, call(n_pos=0), "CAPACITY", "n_pos")
    refused(L, call(sec=None), "ARG", "sections")
    refused(L, call(sec=(1,) * 5), "CAPACITY", "n_axes")
    refused(L, call(sec=(4, 0)), "SHAPE", "sections[1]")
    refused(L, call(sec=(4, 3)), "SHAPE", "sum")
    refused(L, call(sec=(100, 100)), "SHAPE", "sum")
    for base in (1.0, 0.0, -2.0, math.nan, math.inf):
        refused(L, call(base=base), "ARG", "base")
    for bad in (dict(factor=0.0), dict(factor=math.nan), dict(original_len=0.0), dict(low=2.0, high=1.0),
                dict(amplitude=math.inf), dict(low=math.nan)):
        sc = gc.RopeScaling(**{**dict(factor=2.0, original_len=100.0), **bad})
        refused(L, call(scaling=sc), "ARG", "scaling")


def rope(gc, L, x=None, out=None, T=10, H=4, D=64, dtype=1, pos=A[3], table=A[4], n_pos=16, sec=(32,), layout=0):
    x = x if x is not None else heads(gc, A[0])
    out = out if out is not None else heads(gc, A[1])
    return L.gc_rope(ctypes.byref(x), T, H, D, dtype, pos, table, n_pos, i32(*sec), len(sec), layout, ctypes.byref(out), None)


def test_rope_refusals(gc, L):
    refused(L, rope(gc, L, dtype=7), "DTYPE")
    refused(L, rope(gc, L, H=0), "CAPACITY", "heads")
    refused(L, rope(gc, L, H=2000), "CAPACITY", "heads")
    for D in (0, 4, 12, 264):
        refused(L, rope(gc, L, D=D), "SHAPE", "dim")
    refused(L, rope(gc, L, sec=(34,)), "SHAPE", "68")
    refused(L, rope(gc, L, layout=2), "ARG", "layout")
    refused(L, rope(gc, L, T=-1), "CAPACITY", "n_tokens")
    refused(L, rope(gc, L, n_pos=0), "CAPACITY", "n_pos")
    refused(L, rope(gc, L, pos=None), "ARG")
    refused(L, rope(gc, L, table=None), "ARG")
    refused(L, rope(gc, L, table=A[4] + 8), "ALIGN")
    refused(L, rope(gc, L, x=heads(gc, None)), "ARG", "x is null")
    refused(L, rope(gc, L, x=heads(gc, A[0] + 8)), "ALIGN")
    refused(L, rope(gc, L, x=heads(gc, A[0], token=260)), "ALIGN")
    refused(L, rope(gc, L, x=heads(gc, A[0], head=-64)), "SHAPE", "strides")
    refused(L, rope(gc, L, x=heads(gc, A[0], token=1 << 23)), "SHAPE", "strides")
    refused(L, rope(gc, L, out=heads(gc, A[1], head=0)), "SHAPE", "out")       # every head written to one place
    refused(L, rope(gc, L, out=heads(gc, A[1], token=128)), "SHAPE", "out")
    refused(L, rope(gc, L, out=heads(gc, A[0] + 64)), "ALIAS")
    refused(L, rope(gc, L, out=heads(gc, A[0], token=512)), "ALIAS")           # x's place, other strides
    refused(L, rope(gc, L, out=heads(gc, A[4])), "ALIAS", "table")
    assert rope(gc, L, T=0, pos=None, table=None) == 0


def test_norm_refusals(gc, L):
    def call(q=None, k=None, qo=None, ko=None, H=4, Hk=4, T=10, D=64, dtype=1, gq=A[5], gk=A[6], eps=1e-6):
        t = [q or heads(gc, A[0]), k or heads(gc, A[1]), qo or heads(gc, A[7]), ko or heads(gc, A[8])]
        return L.gc_qk_norm_rope(ctypes.byref(t[0]), H, ctypes.byref(t[1]), Hk, T, D, dtype, gq, gk, eps, A[3], A[4], 16,
                                 i32(32), 1, 0, ctypes.byref(t[2]), ctypes.byref(t[3]), None)
    refused(L, call(Hk=0), "CAPACITY")
    refused(L, call(gq=None), "ARG", "gain")
    refused(L, call(gk=A[6] + 4), "ALIGN", "gain")
    for eps in (-1e-6, math.nan, math.inf):
        refused(L, call(eps=eps), "ARG", "eps")
    refused(L, call(qo=heads(gc, A[1])), "ALIAS", "q_out overlaps k")
    refused(L, call(ko=heads(gc, A[7])), "ALIAS", "q_out overlaps k_out")
    refused(L, call(qo=heads(gc, A[5])), "ALIAS", "gain")
    # columns of one buffer of 8 heads a token: apart, or overlapping by a head
    fused = lambda first: heads(gc, A[0] + 128 * first, token=512)
    refused(L, call(q=fused(0), k=fused(4), qo=fused(0), ko=fused(3)), "ALIAS")
    refused(L, call(q=fused(0), k=fused(4), qo=fused(0), ko=fused(4), gq=None), "ARG", "gain")   # apart: only the gain is missed
    assert call(T=0) == 0


def plan_words(gc, L, q_lens, k_lens, H=4, Hk=2, D=64, dtype=1, causal=0):
    info = gc.AttentionInfo()
    n = len(q_lens)
    rc = L.gc_attention_plan(i32(*q_lens), i32(*k_lens), n, H, Hk, D, dtype, causal, ctypes.byref(info), None, 0)
    assert rc == 0, L.gc_last_error().decode()
    words = np.full(info.n_items * 12 + 5, -77, np.int32)
    p = words.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    if info.n_items:
        assert L.gc_attention_plan(i32(*q_lens), i32(*k_lens), n, H, Hk, D, dtype, causal, ctypes.byref(info), p,
                                   info.n_items * 12 - 1) == CODE["CAPACITY"]
    assert (words == -77).all()
    assert L.gc_attention_plan(i32(*q_lens), i32(*k_lens), n, H, Hk, D, dtype, causal, ctypes.byref(info), p,
                               info.n_items * 12) == 0
    assert (words[info.n_items * 12:] == -77).all()
    return info, words[:info.n_items * 12].reshape(-1, 12)


def test_plan_refusals(gc, L):
    info = gc.AttentionInfo()

    def call(q=(3, 4), k=(3, 4), H=4, Hk=2, D=64, dtype=1, n=None, inf=info):
        return L.gc_attention_plan(i32(*q) if q is not None else None, i32(*k) if k is not None else None,
                                   len(q or ()) if n is None else n, H, Hk, D, dtype, 0,
                                   ctypes.byref(inf) if inf is not None else None, None, 0)
    refused(L, call(inf=None), "ARG", "info")
    refused(L, call(H=0), "CAPACITY")
    refused(L, call(Hk=3), "SHAPE", "multiple")
    refused(L, call(Hk=0), "SHAPE")
    refused(L, call(D=60), "SHAPE", "dim")
    refused(L, call(dtype=2), "DTYPE")
    refused(L, call(n=-1), "CAPACITY")
    refused(L, call(q=None, n=2), "ARG")
    refused(L, call(q=(3, -4)), "SHAPE", "sequence 1")
    refused(L, call(k=(-3, 4)), "SHAPE", "sequence 0")
    refused(L, call(q=(2**31 - 1, 1), k=(1, 1), H=1, Hk=1), "CAPACITY")
    refused(L, call(q=(1, 1), k=(2**31 - 1, 2)), "CAPACITY")
    refused(L, call(q=(2**30,), k=(4,), H=64, Hk=1), "CAPACITY")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("D", [8, 64, 128, 256])
@pytest.mark.parametrize("H,Hk", [(1, 1), (8, 2), (64, 1)])
@pytest.mark.parametrize("q_lens,k_lens", [
    ([], []), ([0], [0]), ([0, 5], [9, 0]), ([1], [1]), ([1] * 8, [1, 63, 1000, 4096, 9216, 16384, 24576, 65536]),
    ([1000, 3, 0, 77], [1000, 900, 10, 20]), ([24576], [24576]), ([1], [100000]), ([300], [70000]), ([200], [40]),
    ([1] * 700, [50 + i for i in range(700)])])
def test_plan_items(gc, L, q_lens, k_lens, H, Hk, D, causal, dtype):
    """Every row of every sequence lies in one tile; a tile's parts cover,
    without overlap, all keys that any of its rows sees; slots and counters
    are dealt once and the workspace holds them."""
    info, items = plan_words(gc, L, q_lens, k_lens, H, Hk, D, dtype, causal)
    G, tile = H // Hk, info.tile_rows
    assert (info.heads, info.kv_heads, info.dim, info.dtype, info.causal) == (H, Hk, D, dtype, causal)
    assert (info.total_q, info.total_k) == (sum(q_lens), sum(k_lens))
    at_q, at_k = np.cumsum([0] + list(q_lens)), np.cumsum([0] + list(k_lens))
    tiles, slots, groups = {}, [], {}
    for q0, rows, row0, k0, kb, ke, reach, k_len, slot, slot0, parts, group in items.tolist():
        s = [i for i in range(len(q_lens)) if at_q[i] == q0 and q_lens[i] * G == rows and rows > 0][0]
        assert k0 == at_k[s] and k_len == k_lens[s] and reach == k_lens[s] - q_lens[s] + 1
        assert 0 <= row0 < rows and row0 % tile == 0 and 0 <= kb <= ke <= k_len
        if parts > 1:
            assert 0 <= slot0 <= slot < slot0 + parts <= info.n_slots and 0 <= group < info.n_groups
            slots.append(slot)
            assert groups.setdefault(group, (s, row0)) == (s, row0)
        else:
            assert slot == -1
        tiles.setdefault((s, row0), []).append((kb, ke, parts, slot))
    assert sorted(slots) == list(range(info.n_slots)) and len(groups) == info.n_groups
    want = {(s, r) for s, n in enumerate(q_lens) for r in range(0, n * G, tile)}
    assert set(tiles) == want
    for (s, r), parts in tiles.items():
        parts.sort()
        assert len(parts) == parts[0][2]
        last = (min(r + tile, q_lens[s] * G) - 1) // G
        seen = max(0, min(k_lens[s], last + k_lens[s] - q_lens[s] + 1)) if causal else k_lens[s]
        assert parts[0][0] == 0 and parts[-1][1] >= seen
        for a, b in zip(parts, parts[1:]):
            assert a[1] == b[0] and a[3] < b[3]
    if info.n_slots == 0:
        assert info.workspace_bytes == 0


def test_attention_refusals(gc, L):
    info = gc.AttentionInfo()
    assert L.gc_attention_plan(i32(40), i32(90), 1, 4, 2, 64, 1, 0, ctypes.byref(info), None, 0) == 0

    def call(q=None, k=None, v=None, o=None, lse=A[4], inf=info, items=A[5], scale=0.125, ws=A[6], n=1 << 40):
        t = [q or heads(gc, A[0]), k or heads(gc, A[1], n=2), v or heads(gc, A[2], n=2), o or heads(gc, A[3])]
        return L.gc_attention(*map(ctypes.byref, t), lse, ctypes.byref(inf) if inf is not None else None, items, scale, ws,
                              n, None)
    refused(L, call(inf=None), "ARG", "info")
    refused(L, call(inf=gc.AttentionInfo()), "CAPACITY")
    for name, value in (("kv_heads", 3), ("kv_heads", 0), ("kind", 99), ("tile_rows", 7), ("n_items", -1), ("total_q", -5)):
        other = gc.AttentionInfo.from_buffer_copy(info)
        setattr(other, name, value)
        refused(L, call(inf=other), "ARG", "gc_attention_plan")
    for scale in (0.0, -1.0, math.nan, math.inf):
        refused(L, call(scale=scale), "ARG", "scale")
    refused(L, call(items=None), "ARG", "items")
    refused(L, call(items=A[5] + 4), "ALIGN")
    refused(L, call(lse=A[4] + 2), "ALIGN")
    refused(L, call(k=heads(gc, None)), "ARG", "k is null")
    refused(L, call(v=heads(gc, A[2] + 2)), "ALIGN", "v")
    refused(L, call(o=heads(gc, A[3], token=64)), "SHAPE", "out")
    refused(L, call(o=heads(gc, A[0])), "ALIAS", "q")
    refused(L, call(o=heads(gc, A[1])), "ALIAS", "k")
    refused(L, call(lse=A[2]), "ALIAS", "v")
    refused(L, call(lse=A[3]), "ALIAS")
    refused(L, call(items=A[3]), "ALIAS")
    empty = gc.AttentionInfo()
    assert L.gc_attention_plan(i32(0), i32(90), 1, 4, 2, 64, 1, 0, ctypes.byref(empty), None, 0) == 0
    assert call(inf=empty, items=None, ws=None, n=0) == 0


def test_attention_workspace_refusals(gc, L):
    info = gc.AttentionInfo()
    assert L.gc_attention_plan(i32(1), i32(200000), 1, 4, 2, 64, 1, 0, ctypes.byref(info), None, 0) == 0
    if info.workspace_bytes == 0:
        pytest.skip("no plan of this library splits keys")
    t = [heads(gc, A[0]), heads(gc, A[1], n=2), heads(gc, A[2], n=2), heads(gc, A[3])]

    def call(ws=A[6], n=info.workspace_bytes):
        return L.gc_attention(*map(ctypes.byref, t), A[4], ctypes.byref(info), A[5], 0.125, ws, n, None)
    refused(L, call(ws=None), "ARG", "workspace")
    refused(L, call(n=info.workspace_bytes - 1), "CAPACITY", "workspace")
    refused(L, call(ws=A[6] + 8), "ALIGN")
    refused(L, call(ws=A[1]), "ALIAS")
    refused(L, call(ws=A[3]), "ALIAS")


def test_binding_refusals(gc):
    cpu = torch.zeros((4, 2, 64))
    pos = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros((8, 32, 2))
    gain = torch.ones(64)
    with pytest.raises(ValueError, match="device tensor"):
        gc.gc_rope(cpu, pos, table)
    with pytest.raises(TypeError):
        gc.gc_rope([1.0], pos, table)
    with pytest.raises(ValueError, match="device tensor"):
        gc.gc_qk_norm_rope(cpu, cpu, gain, gain, pos, table)
    with pytest.raises(ValueError, match="axes"):
        gc.gc_rope_table(4, [])
    with pytest.raises(ValueError, match="n_pos"):
        gc.gc_rope_table(0, [4])
    with pytest.raises(ValueError, match="same length"):
        gc.gc_attention_plan([1], [1, 2], 2, 2, 64, torch.float32, device="cpu")
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        gc.gc_attention_plan([1], [1], 2, 2, 64, torch.float16, device="cpu")
    with pytest.raises(ValueError, match="lengths"):
        gc.gc_attention_plan([-1], [1], 2, 2, 64, torch.float32, device="cpu")
    with pytest.raises(gc.GeoCacheError, match="multiple"):
        gc.gc_attention_plan([1], [1], 3, 2, 64, torch.float32, device="cpu")


def test_attention_scale_in_float32(gc, L):
    """A scale that float32 rounds to 0 or to infinity is refused: -inf (a masked score) times 0 is NaN."""
    info = gc.AttentionInfo()
    assert L.gc_attention_plan(i32(40), i32(90), 1, 4, 2, 64, 1, 0, ctypes.byref(info), None, 0) == 0
    t = [heads(gc, A[0]), heads(gc, A[1], n=2), heads(gc, A[2], n=2), heads(gc, A[3])]
    for scale in (1e-60, 5e-324, 3e38, 1e39, 1e300):
        refused(L, L.gc_attention(*map(ctypes.byref, t), A[4], ctypes.byref(info), A[5], scale, A[6], 1 << 40, None), "ARG", "scale")


def test_attention_tokens_that_share_memory(gc, L):
    info = gc.AttentionInfo()
    assert L.gc_attention_plan(i32(40), i32(90), 1, 4, 2, 64, 1, 0, ctypes.byref(info), None, 0) == 0
    for name in "kv":
        t = dict(q=heads(gc, A[0]), k=heads(gc, A[1], n=2), v=heads(gc, A[2], n=2), o=heads(gc, A[3]))
        t[name].token_stride = 56
        refused(L, L.gc_attention(*(ctypes.byref(t[n]) for n in "qkvo"), A[4], ctypes.byref(info), A[5], 0.125, A[6], 1 << 40, None),
                "SHAPE", "token strides of k and v")


def test_attention_plan_without_host_memory(gc, L):
    """A batch whose lists of tiles do not fit the process's memory is refused, and the next plan is as ever."""
    code = """if True:
        import ctypes, resource, sys
        import numpy as np
        import paper_2608_13255_amd as gc
        L = gc.lib()
        n = 1 << 24
        ones = np.ones(n, np.int32)
        p = ones.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        info = gc.AttentionInfo()
        used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
        resource.setrlimit(resource.RLIMIT_AS, (used + (32 << 20), resource.getrlimit(resource.RLIMIT_AS)[1]))
        rc = L.gc_attention_plan(p, p, n, 2, 2, 64, 1, 0, ctypes.byref(info), None, 0)
        text = L.gc_last_error().decode()
        assert L.gc_attention_plan(p, p, 3, 2, 2, 64, 1, 0, ctypes.byref(info), None, 0) == 0
        assert info.n_items == 3
        print(rc, text)
    """
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=Path(__file__).parent.parent)
    assert done.returncode == 0, done.stderr
    assert done.stdout.startswith(f"{CODE['CAPACITY']} ") and "host memory" in done.stdout, done.stdout


def test_norm_eps_in_float32(gc, L):
    """An eps that float32 rounds to 0 would make NaN of heads of zeros (0 / sqrt(eps) is 0), one that it rounds to infinity 0 of all."""
    t = [heads(gc, a) for a in (A[0], A[1], A[7], A[8])]
    for eps in (1e-60, 5e-324, 7e-46, 3.5e38, 1e300):
        refused(L, L.gc_qk_norm_rope(ctypes.byref(t[0]), 4, ctypes.byref(t[1]), 4, 10, 64, 1, A[5], A[6], eps, A[3], A[4], 16,
                                     i32(32), 1, 0, ctypes.byref(t[2]), ctypes.byref(t[3]), None), "ARG", "eps")
    # up to the gain's check (missing here) these are taken
    for eps in (0.0, 1e-45, 1e-6, 3e38):
        refused(L, L.gc_qk_norm_rope(ctypes.byref(t[0]), 4, ctypes.byref(t[1]), 4, 10, 64, 1, None, A[6], eps, A[3], A[4], 16,
                                     i32(32), 1, 0, ctypes.byref(t[2]), ctypes.byref(t[3]), None), "ARG", "gain")
