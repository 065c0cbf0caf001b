"""Edges of the calls on a K/V cache in pages, against the plain fp64 definitions (bounds: as in test_gpu_cache)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_12280_b200 import binding as B_
from paper_2511_12280_b200.cache import PagedCache
from test_gpu_cache import BF, DEV, FP, Pool, check_attention, cu, f64, i32, randn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ protected slots
# columns per key head: few, whose scores go out, and many, whose weights come from a second pass over the keys
@pytest.mark.parametrize("dt,H,kv,dh,block", [(BF, 4, 2, 128, 1), (BF, 4, 1, 128, 16), (BF, 4, 2, 64, 3), (BF, 8, 2, 64, 9), (FP, 4, 2, 64, 3)])
@pytest.mark.parametrize("mode", [B_.WEIGHT_ADD, B_.WEIGHT_SET])
def test_slots_that_are_kept_from_eviction_stay_so_when_weights_are_written(dt, H, kv, dh, block, mode):
    lens, rows = [300, 150, 40], [block, 0, 1]                       # nobody looks at the second request
    P = Pool(lens, 16, kv, dh, dt, seed=31)
    safe = [np.arange(0, n, 7) for n in lens]
    for at, s in zip(P.at, safe):
        P.flat()[2][torch.as_tensor(at[s], device=DEV)] = float("inf")
    had = f64(P.flat()[2])
    q, total = randn((sum(rows), H, dh), dt, 1), sum(rows)
    out = torch.zeros(total, H * dh, dtype=dt, device=DEV)
    ctx = B_.Context(64, 3, H, dh, total, 300)
    ctx.d3tom_attn_cached(P.cache, q, i32(cu(rows)), 3, total, block, 300, dh ** -0.5, mode, None, out)
    k1, v1, w1, t1 = P.flat()
    for b, n in enumerate(lens):
        lo, hi = cu(rows)[b], cu(rows)[b + 1]
        idx = torch.as_tensor(P.at[b], device=DEV)
        _, p, _, _ = co.attend(f64(q[lo:hi]), f64(k1[idx]), f64(v1[idx]), dh ** -0.5)
        want = p.sum(axis=(0, 1)) + (had[P.at[b]] if mode == B_.WEIGHT_ADD else 0.0)
        want[safe[b]] = np.inf
        got = f64(w1)[P.at[b]]
        assert np.array_equal(np.isinf(got), np.isinf(want))
        rest = np.isfinite(want)
        # (2 (dh + 8) 2^-24 sum |q||k| scale is 2e-4 at most: of 128 products of normal numbers, sum |q||k| scale stays below 12)
        assert (np.abs(got[rest] - want[rest]) <= 5e-4 * want[rest]).all()
    budget = [len(s) + 1 for s in safe]
    ctx.d3tom_cache_evict(P.cache, i32(budget), None, 3, 300, P.length)
    for b in range(3):
        kept = t1[torch.as_tensor(P.at[b][: budget[b]], device=DEV)].tolist()
        assert set(safe[b].tolist()) <= set(kept)
    assert ctx.device_status() == 0
