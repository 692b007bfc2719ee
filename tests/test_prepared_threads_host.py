"""Threads that share a prepared rotation or append, without a GPU: each launch has the rows
of its own call, also where another thread calls while it is on its way to the library."""
import threading

import pytest
import torch

from paper_2608_04771_amd import binding as B

BF = torch.bfloat16


@pytest.fixture
def launches(monkeypatch):
    """Tensors of the CPU are taken, and a launch notes the rows that the library would read.  The
    first one lets the other thread go first, if that one can."""
    monkeypatch.setattr(B, "_need_cuda", lambda *ts: None)
    monkeypatch.setattr(B, "_same_gpu", lambda a, b: None)
    started, other, seen = threading.Event(), threading.Event(), []

    def launch(index, fn, *args):
        if not started.is_set():
            started.set()
            other.wait(1.0)
        seen.append([x._obj.data for x in args if isinstance(getattr(x, "_obj", None), B.RecoRows)])
        other.set()
        return B.RECO_OK
    monkeypatch.setattr(B, "_launch", launch)
    return started, seen


def _both(started, call, first, second):
    one = threading.Thread(target=call, args=first)
    one.start()
    assert started.wait(10)
    two = threading.Thread(target=call, args=second)
    two.start()
    for t in (one, two):
        t.join(10)
        assert not t.is_alive()


def _ptrs(*ts):
    return [t.data_ptr() for t in ts]


def test_a_rotation(launches):
    started, seen = launches
    x, y, out = (torch.zeros((1, 2, 3, 4, 64), dtype=BF) for _ in "xyo")
    call = B.PreparedRope(B.Rope(torch.ones(32)), torch.zeros((2, 4), dtype=torch.int32), out)
    _both(started, call, (x,), (y,))
    assert sorted(seen) == sorted([_ptrs(x, out), _ptrs(y, out)])


@pytest.mark.parametrize("queries", [False, True])
def test_an_append(launches, queries):
    started, seen = launches
    cache = B.PagedKVCache(torch.zeros((4, 16, 64), dtype=BF), torch.zeros((4, 16, 64), dtype=BF),
                           torch.zeros((1, 2, 3, 2), dtype=torch.int32), torch.zeros((1, 2, 3), dtype=torch.int32))
    k, v, k2, v2 = (torch.zeros((1, 2, 3, 64), dtype=BF) for _ in "kvkv")
    q, q2, out = (torch.zeros((1, 2, 6, 64), dtype=BF) for _ in "qqo")
    call = B.PreparedPagedAppend(cache, q_out=out if queries else None)
    more, more2 = ([q], [q2]) if queries else ([], [])
    _both(started, call, (k, v, *more), (k2, v2, *more2))
    tail = [out] if queries else []
    assert sorted(seen) == sorted([_ptrs(k, v, *more, *tail), _ptrs(k2, v2, *more2, *tail)])
