"""The cases of perf/operators.py at the edges of their ranges: the library's calls against the plain forms and the 64-bit results."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
_FILE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
_spec = importlib.util.spec_from_file_location("cache_operator_cases", _FILE)
operators = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(operators)


@pytest.fixture
def library(monkeypatch):
    monkeypatch.setattr(operators, "own", True)


@pytest.mark.parametrize("dtype,batch,rows,len_,len_min,weight", [
    ("bf16", 1, 35, 17, 17, "add"), ("bf16", 3, 40, 90, 0, "set"), ("bf16", 1, 9, 4, 4, "none"), ("fp32", 2, 8, 5, 3, "add"), ("bf16", 2, 8, 0, 0, "none")])
def test_blocks_longer_than_what_a_request_has(library, dtype, batch, rows, len_, len_min, weight):
    # a block is as long as its request allows, so a case's rows can be more than the call has
    case = dict(op="attn", dtype=dtype, batch=batch, rows=rows, len=len_, len_min=len_min, heads=8, kv_heads=2, dh=64, page=16, weight=weight)
    got = operators.run(operators.prepare(case, 3))
    for x, y in zip(got, operators.exact(case, 3)):
        # bf16: P and the result are rounded (2^-8 each) over sums of |v| up to 5; fp32: sums of 64 products and of the row's terms
        tol = 2.0 ** -7 * 5 if dtype == "bf16" else 1e-5 * 5
        assert (x.double() - y.double()).abs().max().item() <= tol if x.numel() else x.shape == y.shape
