"""Which stream a call is enqueued on when none is given, on the CPU."""
import pytest
import torch

from paper_2511_12280_b200 import binding as B_


class Library:
    def __init__(self):
        self.streams = {}

    def __getattr__(self, name):
        def call(*args):
            self.streams[name] = args[-1]
            return B_.OK
        return call


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    monkeypatch.setattr(B_, "load", lambda: fake)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    return fake


def test_calls_go_to_the_current_stream_of_the_contexts_device(lib):
    ctx = B_.Context(8, 1, 2, 64, 1, 8, device=3)
    x, n = torch.zeros(8, 128), torch.zeros(8, dtype=torch.int32)
    ctx.d3tom_linear(x, x, None, 1, 1, 1, x)
    ctx.d3tom_ffn(x, x, x, None, 1, 1, 1, x, x)
    ctx.d3tom_proj_qkv(x, x, 1, 1, x, x, x)
    ctx.d3tom_attn_varlen(x, x, x, n, 1, 1, 1, 1.0, x)
    ctx.d3tom_attn_importance(x, x, x, n, n, n, n, 1, 1, 1, 1, 1, 1.0, x, x, n)
    ctx.d3tom_select(x, n, n, n, 1, 1, n, None)
    ctx.d3tom_merge(0, x, n, n, n, n, n, 1, 1, 1, 1, 1, 1, x, n, n, n, n)
    ctx.d3tom_merge_kv(0, x, x, n, n, n, n, n, 1, 1, 1, 1, 1, 1, x, x, n, n, n, n)
    ctx.selftest_wait_timeout(1)
    ctx.d3tom_rope(B_.RopeSpec([1]), x, None, n, 1, 0, x, None)
    del lib.streams["d3tom_create"]
    assert len(lib.streams) == 10 and set(lib.streams.values()) == {1003}


def test_a_stream_that_is_given_is_taken(lib):
    ctx, x = B_.Context(8, 1, 2, 64, 1, 8, device=3), torch.zeros(8, 128)
    ctx.d3tom_linear(x, x, None, 1, 1, 1, x, stream=77)
    assert lib.streams["d3tom_linear"] == 77
