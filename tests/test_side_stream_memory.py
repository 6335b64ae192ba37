"""Where the binding takes memory from for a call on an explicit stream (torch's streams replaced, no GPU)."""
import pytest
import torch


@pytest.fixture
def gc():
    import paper_2608_13255_amd as gc
    return gc


# calls that allocate before they find that their input is not on a device
CALLS = {
    "posmap_downsample": lambda gc, s: gc.gc_posmap_downsample(torch.zeros((1, 4, 4, 3)), 2, stream=s),
    "posmap_bbox": lambda gc, s: gc.gc_posmap_bbox(torch.zeros((1, 2, 4, 4, 3)), stream=s),
    "coverage_init": lambda gc, s: gc.gc_coverage_init(torch.zeros((1, 2, 4, 4, 3)), stream=s),
    "coverage_update": lambda gc, s: gc.gc_coverage_update(torch.zeros(4, dtype=torch.int32),
                                                           torch.zeros((1, 2, 4, 4), dtype=torch.uint8), [0], 1, stream=s),
    "index_foreground": lambda gc, s: gc.gc_index_foreground(torch.zeros((1, 2, 4, 4, 3)), stream=s),
    "transport_step": lambda gc, s: gc.gc_transport_step(torch.zeros((1, 2, 4, 4, 8)), torch.zeros((1, 1, 4, 4, 8)),
                                                         torch.zeros((1, 1, 4, 4, 1), dtype=torch.int32),
                                                         torch.zeros((1, 1, 4, 4, 1, 2)), [0], stream=s),
    "rope_table": lambda gc, s: gc.gc_rope_table(8, [4], device="cpu", stream=s),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("side", [True, False])
def test_memory_comes_from_the_stream_that_works_on_it(gc, monkeypatch, name, side):
    current, places = ["here"], []
    real = torch.empty

    def set_stream(stream):
        current[0] = stream

    def empty(*args, **kwargs):
        places.append(current[0])
        return real(*args, **kwargs)

    monkeypatch.setattr(torch.cuda, "set_stream", set_stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[0])
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(gc, "_side_stream", lambda stream: stream if side else None)
    with pytest.raises(ValueError, match="device tensor"):
        CALLS[name](gc, "there")
    assert places and set(places) == {"there" if side else "here"}
    assert current == ["here"]
