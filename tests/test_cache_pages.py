"""Pages and lengths that PagedCache keeps on the host, on the CPU: a stand-in for the library says what the calls say."""
import types

import pytest
import torch

from paper_2511_12280_b200 import binding as B_
from paper_2511_12280_b200 import cache as cache_module

BF = torch.bfloat16
H, KV, DH, PAGE = 4, 2, 64, 8


class Library:
    def __init__(self):
        self.calls, self.status = [], B_.OK

    def d3tom_create(self, *args):
        return B_.OK

    def d3tom_status_string(self, status):
        return b"refused"

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or self.status


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    on_cpu = types.SimpleNamespace(**{n: getattr(torch, n) for n in ("zeros", "zeros_like", "as_tensor", "from_numpy", "tensor", "float32", "int32")},
                                   device=lambda kind, index: torch.device("cpu"), dtype=torch.dtype)
    monkeypatch.setattr(cache_module, "torch", on_cpu)
    monkeypatch.setattr(B_, "load", lambda: fake)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(B_, "_raw_stream", lambda stream, device: 0)
    return fake


def paged(pages=12):
    return cache_module.PagedCache(3, H, KV, DH, BF, pages, PAGE, max_rows=64, max_length=40, max_scored_rows=8)


def rows(n, heads=KV, dt=BF):
    return torch.zeros(n, heads, DH, dtype=dt)


def state(c):
    return c.lengths_h[:], c.length.tolist(), c.table_h.tolist(), c.table.tolist(), c.free[:]


def put(c, n):
    c.append(n, rows(sum(n)), rows(sum(n)), None)


def check_pages(c):
    """Every page belongs to one request or is free, and the device has what the host has."""
    held = [int(p) for b, n in enumerate(c.lengths_h) for p in c.table_h[b, : -(-n // PAGE)]]
    assert sorted(held + c.free) == list(range(12)) and c.length.tolist() == c.lengths_h and c.table.tolist() == c.table_h.tolist()
    for b, n in enumerate(c.lengths_h):
        assert (c.table_h[b, -(-n // PAGE):] == -1).all()


def test_pages_follow_the_lengths(lib):
    c = paged()
    for step in (lambda: put(c, [20, 0, 3]), lambda: put(c, [1, 8, 6]), lambda: c.drop_last([1, 8, 0]), lambda: c.evict([9, 5, 8]),
                 lambda: put(c, [0, 40, 0])):
        step()
        check_pages(c)
    assert c.lengths_h == [9, 40, 8]


@pytest.mark.parametrize("fault", ["status", "type", "short", "full", "long", "rows"])
def test_a_refused_append_changes_nothing(lib, fault):
    c = paged()
    put(c, [20, 0, 3])
    c.evict([9, 0, 3])
    before, n = state(c), [3, 9, 5]
    if fault == "status":
        lib.status = B_.ERR_WORKSPACE
    with pytest.raises((RuntimeError, TypeError)):
        if fault == "full":
            c.append([31, 40, 37], rows(108), rows(108), None)
        elif fault == "long":
            c.append([32, 0, 0], rows(32), rows(32), None)
        else:
            c.append(n, rows(17, dt=torch.float32) if fault == "type" else rows(17), rows(16 if fault == "short" else 17),
                     torch.zeros(2, dtype=torch.int32) if fault == "rows" else None)
    assert state(c) == before
    check_pages(c)
    lib.status = B_.OK
    put(c, n)
    assert c.lengths_h == [12, 9, 8]
    check_pages(c)


@pytest.mark.parametrize("bad", [[21, 0, 0], [0, 1, 0], [1, 0], [0, 0, 0, 0], [-1, 0, 0]])
def test_rows_that_are_not_there_are_not_dropped(lib, bad):
    c = paged()
    put(c, [20, 0, 3])
    before = state(c)
    with pytest.raises(ValueError):
        c.drop_last(bad)
    assert state(c) == before


@pytest.mark.parametrize("bad", [[3, -1, 2], [4, 0], [1, 1, 1, 1]])
def test_rows_of_every_request_and_none_negative(lib, bad):
    c = paged()
    put(c, [20, 10, 3])
    before, n = state(c), len(lib.calls)
    for call in (lambda: c.append(bad, rows(4), rows(4), None), lambda: c.attend(bad, rows(4, H), torch.zeros(4, H * DH, dtype=BF))):
        with pytest.raises(ValueError):
            call()
        assert state(c) == before and len(lib.calls) == n


@pytest.mark.parametrize("bad", [[4, 0], [1, 1, 1, 1]])
def test_a_budget_of_every_request(lib, bad):
    c = paged()
    put(c, [20, 10, 3])
    before, n = state(c), len(lib.calls)
    with pytest.raises(ValueError):
        c.evict(bad)
    assert state(c) == before and len(lib.calls) == n


def test_a_refused_eviction_changes_nothing(lib):
    c = paged()
    put(c, [20, 10, 3])
    before = state(c)
    lib.status = B_.ERR_INVALID_ARG
    with pytest.raises(RuntimeError):
        c.evict([1, 1, 1])
    assert state(c) == before
