"""What a refused or failed call of the layers over a paged cache leaves behind (no GPU)."""

import sys

import pytest
import torch

from paper_2607_20940_amd import mssa
from paper_2607_20940_amd.paged import PagedStreams


def _streams(**kw):
    return PagedStreams(**dict(dict(layers=1, hidden=64, q_heads=4, kv_heads=2, head_dim=64, pages=400, page_tokens=8,
                                    max_stream_pages=200, max_tokens=600, max_batch=3, adapters=2, rank=8, device="cpu"),
                               **kw))


def _state(p):
    """All that a pass changes: page accounts, streams, the open pass's sizes and tensors."""
    places = [getattr(p, n).tolist() for n in ("chunk_begin", "kv_len", "adapter", "table", "positions") if p.batch]
    made = [id(getattr(p, n, None)) for n in ("places", "workspace", "project", "append", "attend")]
    return list(p.free), {s: [list(v[0]), *v[1:]] for s, v in p.streams.items()}, p.batch, getattr(p, "tokens", None), places, made


class _Torch:
    """torch, but for one function that raises as an allocation does that finds no memory."""

    def __init__(self, name):
        self.name = name

    def __getattr__(self, name):
        if name != self.name:
            return getattr(torch, name)

        def none(*args, **kw):
            raise torch.OutOfMemoryError("no memory")

        return none


@pytest.mark.parametrize("opened", [False, True])
@pytest.mark.parametrize("name", ["empty", "tensor"])
def test_passes_that_find_no_memory_change_nothing(monkeypatch, name, opened):
    p = _streams()
    p.open("a")
    p.open("b", 1)
    if opened:
        p.begin([("a", 1), ("b", 3)])
    p.workspace = torch.empty(0, dtype=torch.uint8)  # any pass has to make one
    before = _state(p)
    with monkeypatch.context() as m:
        m.setitem(sys.modules, "torch", _Torch(name))
        with pytest.raises(torch.OutOfMemoryError):
            p.begin([("b", 2), ("a", 300)])
    assert _state(p) == before
    # and the same pass begins where there is memory
    p.begin([("b", 2), ("a", 300)])
    held = {"a": 301, "b": 5} if opened else {"a": 300, "b": 2}
    assert {s: v[1] for s, v in p.streams.items()} == held
    assert p.kv_len.tolist() == [held["b"], held["a"]] and p.batch == 2 and p.tokens == 302
    assert p.positions.tolist() == list(range(held["b"] - 2, held["b"])) + list(range(held["a"] - 300, held["a"]))
    pages = [g for v in p.streams.values() for g in v[0]]
    assert len(pages) == sum(-(-n // 8) for n in held.values()) and sorted(p.free + pages) == list(range(400))


@pytest.mark.parametrize("kw", [dict(freqs=torch.zeros(12), rotate_dims=24),  # halves of 12 pairs
                                dict(freqs=torch.zeros(32), axis_pairs=[16, 15]),
                                dict(freqs=torch.zeros(32), axis_pairs=[33, -1])])
def test_passes_that_the_append_refuses_change_nothing(kw):
    p = _streams(**kw)
    p.open("a")
    before = _state(p)
    for n in (0, 9):
        with pytest.raises(mssa.MssaError):
            p.begin([("a", n)])
        assert _state(p) == before


@pytest.mark.parametrize("adapters,refused", [(0, (0, 1, -2)), (1, (1, -2)), (2, (2, -2))])
def test_adapters_that_are_not_there_are_refused(adapters, refused):
    p = _streams(adapters=adapters)
    for j in refused:
        with pytest.raises(ValueError):
            p.open("a", j)
    assert p.streams == {}
    for j in range(-1, adapters):
        p.open(j, j)
    assert [v[3] for v in p.streams.values()] == list(range(-1, adapters))


def _opened(monkeypatch, **kw):
    """Layers with weights and an open pass of 5 tokens, and the names of the library calls that a pass makes."""
    bf, calls = torch.bfloat16, []
    p = _streams(adapters=0, **kw)
    p.init_layer(0, torch.zeros(512, 64, dtype=bf))
    p.open("a")
    p.begin([("a", 5)])
    for name in ("mssa_adapter_project", "mssa_paged_append", "mssa_paged_attention"):
        monkeypatch.setattr(mssa, name, lambda *a, _name=name, **k: calls.append(_name))
    return p, calls, torch.zeros(5, 64, dtype=bf), torch.zeros(5, 4, 64, dtype=bf), torch.zeros(4, 5)


def test_a_refused_layer_enqueues_nothing(monkeypatch):
    p, calls, x, out, lse = _opened(monkeypatch, layers=2)
    shifted = torch.zeros(5 * 256 + 8, dtype=torch.bfloat16)
    shifted = next(s for s in (shifted[i:i + 5 * 256].view(5, 4, 64) for i in (1, 2)) if s.data_ptr() % 16)
    for args in ((0, x, out, lse, None, out, None), (0, x, out, lse, None, None, lse), (1, x, out),
                 (0, x, shifted), (0, x, out, None, None, shifted, lse), (0, x, p.q[:5]), (0, x, p.k_pages[0].view(-1)[:1280].view(5, 4, 64))):
        with pytest.raises(ValueError):
            p.layer_pass(*args, stream=0)
        assert calls == []
    p.layer_pass(0, x, out, lse, prior_out=out, prior_lse=lse, stream=0)
    assert calls == ["mssa_adapter_project", "mssa_paged_append", "mssa_paged_attention"]


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Their addresses are none of the device's."""
    bf = torch.bfloat16
    w, bias, a, b = torch.zeros(512, 64, dtype=bf), torch.zeros(512, dtype=bf), torch.zeros(2, 8, 64, dtype=bf), torch.zeros(2, 512, 8, dtype=bf)
    scale = torch.zeros(2)
    p = _streams()
    for i in range(5):
        given = [w, bias, a, b, scale]
        given[i] = given[i].to("meta")
        with pytest.raises(ValueError):
            p.init_layer(0, *given)
    assert p.weights == [None]
    with pytest.raises(ValueError):
        _streams(freqs=torch.zeros(32, device="meta"))
    p, calls, x, out, lse = _opened(monkeypatch, freqs=torch.zeros(32))
    given = (x, out, lse, torch.zeros(1, 5, dtype=torch.int32), torch.zeros_like(out), torch.zeros_like(lse))
    for i in range(6):
        with pytest.raises(ValueError):
            p.layer_pass(0, *(t.to("meta") if i == j else t for j, t in enumerate(given)), stream=0)
    assert calls == []
    p.layer_pass(0, *given, stream=0)
    assert len(calls) == 3


def test_the_package_names_the_module():
    import paper_2607_20940_amd

    assert "paged" in paper_2607_20940_amd.__all__
