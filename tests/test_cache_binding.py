"""What the binding refuses of the calls on a cache in pages before the library sees it, on the CPU: a stand-in for the library
records the calls that reach it."""
import pytest
import torch

from paper_2511_12280_b200 import binding as B_

BF, FP = torch.bfloat16, torch.float32
H, KV, DH, PAGE = 4, 2, 64, 8


class Library:
    """Takes every call and says that it is done."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: B_.OK if name == "d3tom_create" else self.calls.append(name) or B_.OK


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    monkeypatch.setattr(B_, "load", lambda: fake)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(B_, "_raw_stream", lambda stream, device: 0)
    return fake


def context(head_dim=DH, tokens=16, deciders=8):
    return B_.Context(tokens, 2, H, head_dim, deciders, 32)


def i32(*a):
    return torch.tensor(a, dtype=torch.int32)


def cache(kv=KV, dh=DH, dt=BF):
    k = torch.zeros(4, PAGE, kv, dh, dtype=dt)
    return B_.Cache(k, torch.zeros_like(k), torch.zeros(4, PAGE), torch.zeros(4, PAGE, dtype=torch.int32), i32(0, 1, 2, 3).view(2, 2), i32(9, 3))


def rows(n, heads, dt=BF, dh=DH):
    return torch.zeros(n, heads, dh, dtype=dt)


def append(ctx, c={}, q=None, k=None, v=None, first=None, q_out=None, n=3):
    ctx.d3tom_cache_append(cache(**c), None, rows(n, H) if q is None else q, rows(n, KV) if k is None else k, rows(n, KV) if v is None else v,
                           None, None, first, i32(0, 2, n), 2, n, rows(n, H) if q_out is None else q_out)


def attend(ctx, c={}, q=None, out=None, row_weight=None, n=3, mode=B_.WEIGHT_ADD):
    ctx.d3tom_attn_cached(cache(**c), rows(n, H) if q is None else q, i32(0, 2, n), 2, n, n, 9, 0.1, mode, row_weight,
                          torch.zeros(n, H * DH, dtype=BF) if out is None else out)


def evict(ctx, c={}):
    ctx.d3tom_cache_evict(cache(**c), i32(4, 4), None, 2, 9, i32(0, 0))


def rope(ctx, q=None, k=None, q_out=None, k_out=None, n=3):
    ctx.d3tom_rope(B_.RopeSpec([8]), rows(n, H) if q is None else q, rows(n, KV) if k is None else k, torch.zeros(n, 1, dtype=torch.int32), n, KV,
                   rows(n, H) if q_out is None else q_out, rows(n, KV) if k_out is None else k_out)


BAD = [
    # a cache of another head size than the context's
    (append, dict(c=dict(dh=128)), ValueError), (attend, dict(c=dict(dh=32)), ValueError), (evict, dict(c=dict(dh=128)), ValueError),
    # fp32 arrays of another type, or too short
    (append, dict(first=torch.zeros(3, dtype=torch.float64)), TypeError), (append, dict(first=torch.zeros(3, dtype=BF)), TypeError),
    (append, dict(first=torch.zeros(2)), TypeError), (attend, dict(row_weight=torch.zeros(3, dtype=torch.float64)), TypeError),
    (attend, dict(row_weight=torch.zeros(3, dtype=torch.int32)), TypeError), (attend, dict(row_weight=torch.zeros(2)), TypeError),
    # rows that are not all there: of the call, of the heads, of the head size
    (append, dict(q=rows(2, H)), TypeError), (append, dict(k=rows(2, KV)), TypeError), (append, dict(v=rows(3, KV - 1)), TypeError),
    (append, dict(q_out=rows(3, H, dh=32)), TypeError), (append, dict(c=dict(kv=4)), TypeError), (attend, dict(q=rows(3, H - 1)), TypeError),
    (attend, dict(out=torch.zeros(2, H * DH, dtype=BF)), TypeError), (rope, dict(q=rows(2, H)), TypeError), (rope, dict(k=rows(3, 1)), TypeError),
    (rope, dict(q_out=rows(1, H)), TypeError), (rope, dict(k_out=rows(2, KV)), TypeError),
    # rows of two types
    (append, dict(v=rows(3, KV, FP)), TypeError), (attend, dict(out=torch.zeros(3, H * DH)), TypeError), (rope, dict(q=rows(3, H, FP)), TypeError),
    (rope, dict(k=rows(3, KV, FP)), TypeError), (rope, dict(q_out=rows(3, H, FP)), TypeError), (rope, dict(k_out=rows(3, KV, FP)), TypeError),
]


@pytest.mark.parametrize("call,args,error", BAD)
def test_what_would_be_read_or_written_out_of_range_is_refused(lib, call, args, error):
    with pytest.raises(error):
        call(context(), **args)
    assert lib.calls == []


def test_calls_that_fit_reach_the_library(lib):
    ctx = context()
    append(ctx)
    append(ctx, first=torch.zeros(3))
    append(ctx, q=rows(5, H), k=rows(4, KV), first=torch.zeros(9))            # rows behind the last request are the caller's
    attend(ctx, row_weight=torch.zeros(3))
    attend(ctx, out=rows(3, H), mode=B_.WEIGHT_NONE)
    rope(ctx)
    rope(ctx, q=rows(4, H))
    evict(ctx)
    assert lib.calls == ["d3tom_cache_append"] * 3 + ["d3tom_attn_cached"] * 2 + ["d3tom_rope"] * 2 + ["d3tom_cache_evict"]


def test_what_exceeds_the_context_is_left_to_the_library(lib):
    # which says D3TOM_ERR_WORKSPACE, whatever was handed over
    append(context(tokens=2), q=rows(1, H))
    attend(context(tokens=2), q=rows(1, H))
    attend(context(deciders=2), q=rows(1, H))
    rope(context(tokens=2), q=rows(1, H))
    assert len(lib.calls) == 4

