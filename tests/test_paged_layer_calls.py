"""What the layers over a paged cache refuse, and their page accounts (no GPU)."""

import pytest
import torch

from paper_2607_20940_amd import mssa
from paper_2607_20940_amd.paged import PagedStreams


def _streams(**kw):
    return PagedStreams(**dict(dict(layers=1, hidden=64, q_heads=4, kv_heads=2, head_dim=64, pages=10, page_tokens=8,
                                    max_stream_pages=6, max_tokens=60, max_batch=3, adapters=2, rank=8, device="cpu"), **kw))


def test_pages_are_counted():
    p = _streams()
    for s in "abc":
        p.open(s)
    p.begin([("a", 17), ("b", 1)])
    assert [len(p.streams[s][0]) for s in "abc"] == [3, 1, 0] and len(p.free) == 6
    p.begin([("a", 7), ("c", 0)])
    assert len(p.streams["a"][0]) == 3 and p.kv_len.tolist() == [24, 0] and p.chunk_begin.tolist() == [0, 7, 7]
    assert p.positions.tolist() == list(range(17, 24))
    p.drop("a", 16)
    assert p.streams["a"][1:3] == [8, 16] and len(p.free) == 8
    p.begin([("a", 1)])
    assert p.positions.tolist() == [24] and p.kv_len.tolist() == [9]
    p.close("a")
    p.close("b")
    assert sorted(p.free) == list(range(10))
    assert len({*p.free}) == 10


def test_refused_passes_change_nothing():
    p = _streams()
    p.open("a")
    p.open("b", 1)
    p.begin([("a", 40)])
    before = (list(p.free), {s: list(map(str, v)) for s, v in p.streams.items()})
    for bad in ([], [("x", 1)], [("a", 1), ("a", 1)], [("a", 61)], [("a", 20)], [("b", -1)], [("a", 0)] * 4):
        with pytest.raises(ValueError):
            p.begin(bad)
    with pytest.raises(RuntimeError):
        p.begin([("b", 47)])
    assert before == (p.free, {s: list(map(str, v)) for s, v in p.streams.items()})
    for tokens in (4, 48, -8):
        with pytest.raises(ValueError):
            p.drop("a", tokens)
    with pytest.raises(ValueError):
        p.open("a")
    for adapter in (2, -2):
        with pytest.raises(ValueError):
            p.open("z", adapter)


def test_passes_that_the_library_refuses_change_nothing():
    p = _streams(rank=300)
    p.open("a")
    with pytest.raises(mssa.MssaError):
        p.begin([("a", 9)])
    assert len(p.free) == 10 and p.streams["a"][:2] == [[], 0] and p.batch is None


def test_tensors_of_other_types_and_shapes_are_refused():
    bf = torch.bfloat16
    p = _streams()
    w, a, b = torch.zeros(512, 64, dtype=bf), torch.zeros(2, 8, 64, dtype=bf), torch.zeros(2, 512, 8, dtype=bf)
    for bad in ((w.float(), None, a, b), (w[:500], None, a, b), (w, torch.zeros(512), a, b), (w, None, None, b), (w, None, a, b[:1])):
        with pytest.raises(ValueError):
            p.init_layer(0, *bad)
    with pytest.raises(ValueError):
        p.init_layer(0, w, None, a, b, torch.zeros(3))
    p.init_layer(0, w, None, a, b)
    x, out = torch.zeros(5, 64, dtype=bf), torch.zeros(5, 4, 64, dtype=bf)
    with pytest.raises(ValueError):
        p.layer_pass(0, x, out)  # no pass is open
    p.open("a")
    p.begin([("a", 5)])
    for args in ((x.float(), out), (x[:4], out), (x, out[:, :3]), (x, out, torch.zeros(4, 5, dtype=bf)),
                 (x, out, None, torch.zeros(2, 5, dtype=torch.int32))):
        with pytest.raises(ValueError):
            p.layer_pass(0, *args)
    with pytest.raises(ValueError):
        _streams(freqs=torch.zeros(31))
    q = _streams(freqs=torch.zeros(32), axis_pairs=[16, 16])
    q.open("a")
    q.begin([("a", 5)])
    with pytest.raises(ValueError):
        q.layer_pass(0, x, out)
