"""When a block's weights are laid out in 8 bits again: what other threads and
streams see of it (the operators replaced by ones on the CPU, no GPU)."""
import copy
from types import SimpleNamespace

import pytest
import torch

from paper_2608_13255_amd import multiview

NAMES = ("w_qkv", "w_out", "w_in", "w_down")


def block_with(numbers):
    """A block without its construction; weight `name` holds numbers[name]."""
    block = object.__new__(multiview.MultiViewBlock)
    block.width, block.heads, block.kv_heads, block.dim, block.hidden = 16, 2, 1, 16, 32
    block.dtype, block.eps, block.act, block.gated = torch.float32, 1e-6, 1, False
    block.foreground = torch.ones((1, 1, 1, 1), dtype=torch.bool)
    block.eight_bits, block._captured = None, {}
    for name in NAMES:
        setattr(block, name, torch.full((1, 1), float(numbers[name])))
        setattr(block, "b" + name[1:], None)
    block.q_gain = block.k_gain = block.attention_gain = block.feed_gain = torch.ones(1)
    return block


class Stream:
    cuda_stream = 77

    def __init__(self, at_synchronize=lambda: None):
        self.at_synchronize = at_synchronize

    def synchronize(self):
        self.at_synchronize()


@pytest.fixture
def quantized(monkeypatch):
    monkeypatch.setattr(multiview, "gc_quantize_rows", lambda w: (w.clone(), torch.ones(1)))


def test_weights_are_published_when_they_are_complete(monkeypatch, quantized):
    block = block_with(dict.fromkeys(NAMES, 1))
    seen = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream(lambda: seen.append(block.eight_bits)))
    block.lay_out_in_8_bits()
    first = block.eight_bits
    assert seen == [None] and set(first) == set(NAMES)
    block.lay_out_in_8_bits()
    assert seen[1] is first and block.eight_bits is not first


def test_a_call_keeps_the_weights_it_began_with(monkeypatch, quantized):
    block = block_with(dict.fromkeys(NAMES, 1))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    block.lay_out_in_8_bits()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(block, "_tokens", lambda x, views, weights: (SimpleNamespace(), torch.zeros(3, 32)), raising=False)
    monkeypatch.setattr(block, "_attend", lambda qkv, s: torch.zeros(3, 32), raising=False)
    monkeypatch.setattr(block, "_spread", lambda y, x, s: y, raising=False)
    monkeypatch.setattr(multiview, "gc_add_rms_norm", lambda x, **more: (x, torch.ones(3), x))
    used = []

    def product(x, w, bias, **more):
        used.append(float(w))
        for name in NAMES:                       # another thread, between two products
            getattr(block, name).add_(1)
        block.lay_out_in_8_bits()
        return torch.zeros(3, 32)

    monkeypatch.setattr(multiview, "gc_linear", product)
    block(torch.zeros(3, 32), [0])
    assert used == [1, 1, 1, 1]
    block(torch.zeros(3, 32), [0])
    assert used[4:] == [5, 5, 5, 5]


def test_weights_are_known_on_each_stream_that_reads_them(monkeypatch):
    """Each stream that reads them is told to the allocator once; the one that they were made on needs no telling."""
    told = []

    class Tensor:
        device = torch.device("cuda:0")

        def record_stream(self, stream):
            told.append((id(self), stream.cuda_stream))

    pairs = {name: (Tensor(), Tensor()) for name in NAMES}
    rows = multiview.EightBitWeights(pairs)
    rows.known_streams.add(77)
    home, other = Stream(), Stream()
    other.cuda_stream = 78
    for stream in (home, other, home, other):
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: stream)
        rows.used_here()
    assert sorted(told) == sorted((id(t), 78) for pair in pairs.values() for t in pair)


def test_a_copy_is_known_on_no_stream():
    rows = multiview.EightBitWeights({"w_in": (torch.zeros(2), torch.ones(1))})
    rows.known_streams.add(77)
    other = copy.deepcopy(rows)
    assert not other.known_streams and rows.known_streams == {77}
    assert torch.equal(other["w_in"][0], rows["w_in"][0]) and other["w_in"][0] is not rows["w_in"][0]


def test_what_a_graph_reads_stays(monkeypatch):
    """A slice or weights that a captured call reads are kept with the layer, those of other calls are not."""
    block = block_with(dict.fromkeys(NAMES, 1))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    shared = [multiview.EightBitWeights({"w_in": (torch.zeros(2), torch.ones(1))}) for _ in range(2)]
    for s in shared:
        s.known_streams.add(Stream.cuda_stream)
    for capturing, s in ((False, shared[0]), (True, shared[1]), (True, shared[1])):
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
        block._uses(s)
    assert [c is shared[1] for c in block._captured.values()] == [True]
