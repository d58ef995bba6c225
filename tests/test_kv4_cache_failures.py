"""Kv4Cache: a call that fails on its way, wherever that is, leaves the pages and tokens of all sequences as they were, on the host and in
what the GPU reads.  CPU: the entry points are stood in for."""
import pytest
import torch

from paper_2604_03260_b200 import binding as fb
from paper_2604_03260_b200.kv4_cache import Kv4Cache


class Lost(RuntimeError):
    pass


def lose(*args, **kw):
    raise Lost


@pytest.fixture
def layer(monkeypatch):
    """sequence 0 has 20 tokens in pages 0 and 1, sequence 1 the same (shared), 2 has 16 in page 3, 3 nothing; page 2 is a hole"""
    c = Kv4Cache(4, 4, 2, 64, 4, 2, 16, 64, 8, 16, device="cpu")
    for name in ("focus_kv4_copy_pages", "focus_kv4_append", "focus_kv4_decode_step", "focus_kv4_read"):
        monkeypatch.setattr(fb, name, lambda *a, **kw: None)
    c.reserve([20, 16, 0, 0])
    c.reserve([0, 0, 16, 0])
    c.free(1)
    c.fork(0, 1)
    assert c.held == [[0, 1], [0, 1], [3], []] and c.refs == [2, 2, 0, 1, 0, 0, 0, 0]
    return c


def host(c):
    return list(c.refs), [list(p) for p in c.held], list(c.tokens)


def on_gpu(c):
    """what a kernel would see: the pages of every sequence, by its length"""
    return [c.table[b, :-(-n // c.P)].tolist() for b, n in enumerate(c.lens.tolist())], c.lens.tolist()


def agree(c):
    return on_gpu(c) == (c.held, c.tokens)


k = torch.zeros((4, 2, 3, 64), dtype=torch.bfloat16)
mk = torch.zeros((8, 3), dtype=torch.int32)
CALLS = {"reserve": lambda c: c.reserve([1, 0, 0, 2]), "append": lambda c: c.append(k, k, mk, [1, 3, 0, 2]), "fork": lambda c: c.fork(0, 3),
         "free": lambda c: c.free(0), "compact": lambda c: c.compact()}


@pytest.mark.parametrize("call,where", [(c, w) for c in CALLS for w in ("_push", "_move", "copy_pages") if w == "_push" or c not in ("fork", "free")])
def test_a_failure_leaves_everything_as_it_was(layer, monkeypatch, call, where):
    before = host(layer), on_gpu(layer)
    with monkeypatch.context() as m:
        m.setattr(*((fb, "focus_kv4_copy_pages", lose) if where == "copy_pages" else (layer, where, lose)))
        with pytest.raises(Lost):
            CALLS[call](layer)
        assert (host(layer), on_gpu(layer)) == before
    CALLS[call](layer)                       # and as if nothing had been: the call goes through
    assert agree(layer) and host(layer) != before[0]


def test_table_and_lengths_change_together(layer, monkeypatch):
    """a copy to the GPU that fails leaves neither of them new"""
    before = on_gpu(layer)
    copies = []
    real = torch.Tensor.copy_

    def second_fails(self, *a, **kw):
        copies.append(self.shape)
        if len(copies) > 1:
            raise Lost
        return real(self, *a, **kw)
    with monkeypatch.context() as m:
        m.setattr(torch.Tensor, "copy_", second_fails)
        try:
            layer.free(0)
        except Lost:
            pass
    assert on_gpu(layer) == before or agree(layer)


def test_a_refused_append_whose_restoration_fails_too(layer, monkeypatch):
    """the next call that reads the pages brings table and lengths back first"""
    before = host(layer)
    pushes, real = [], layer._push

    def second_fails(stream=None):
        pushes.append(1)
        if len(pushes) == 2:
            raise Lost
        real(stream)
    monkeypatch.setattr(layer, "_push", second_fails)
    monkeypatch.setattr(fb, "focus_kv4_append", lose)
    with pytest.raises(Lost):
        layer.append(k, k, mk)
    assert host(layer) == before and len(pushes) == 2
    seen = []
    monkeypatch.setattr(fb, "focus_kv4_decode_step", lambda *a, **kw: seen.append(agree(layer)))
    monkeypatch.setattr(fb, "focus_kv4_read", lambda *a, **kw: seen.append(agree(layer)))
    layer.decode(None, None, None, None)
    layer.read(k, k)
    assert seen == [True, True] and len(pushes) == 3


def test_a_sequence_that_is_none(layer):
    before = host(layer), on_gpu(layer)
    for call in (lambda: layer.fork(4, 3), lambda: layer.fork(0, 4), lambda: layer.free(4)):
        with pytest.raises(IndexError):
            call()
        assert (host(layer), on_gpu(layer)) == before
