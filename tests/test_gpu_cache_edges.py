"""Edges of the calls on a K/V cache in pages, against the plain fp64 definitions (bounds: as in test_gpu_cache)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_12280_b200 import binding as B_
from paper_2511_12280_b200.cache import PagedCache
from test_gpu_cache import BF, DEV, FP, Pool, check_attention, cu, f64, i32, randn

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ angles
@pytest.mark.parametrize("theta,turns", [(1e4, 2.0 ** -32), (1e6, 2.0 ** -32), (1.5, 2.0 ** -28)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_angles_of_far_positions(theta, turns, neighbours):
    # the pair (1, 0) becomes (cos, sin), which are small themselves near quarter and half turns: there the angle's own error is seen.
    # Bound: the angle, 2 units of the last digit (sincospif 1, the rest of the angle 1/2, both at most 2^-23 of the value)
    rows, H, dh = 2048, 1, 128
    pos = np.random.default_rng(7).integers(-2 ** 31, 2 ** 31, (rows, 1))
    pos[:4, 0] = [0, 1, 2 ** 31 - 1, -2 ** 31]
    x = torch.zeros(rows, H, dh, device=DEV)
    x[..., 0::2] = 1.0
    if not neighbours:
        x = torch.cat([torch.ones(rows, H, dh // 2, device=DEV), torch.zeros(rows, H, dh // 2, device=DEV)], dim=-1).contiguous()
    spec = B_.RopeSpec([64], theta, B_.PAIR_NEIGHBOURS if neighbours else B_.PAIR_HALVES)
    out = torch.empty_like(x)
    B_.Context(rows, 1, H, dh, 1, 1).d3tom_rope(spec, x, None, i32(pos), rows, 0, out, None)
    y = f64(out)[:, 0]
    c, s = (y[:, 0::2], y[:, 1::2]) if neighbours else (y[:, : dh // 2], y[:, dh // 2 :])
    ang = co.rope_angles(pos, [64], theta, False)
    assert (np.abs(np.sin(ang)) < 0.01).sum() > 500 and (np.abs(np.cos(ang)) < 0.01).sum() > 500
    for got, want in ((c, np.cos(ang)), (s, np.sin(ang))):
        assert (np.abs(got - want) <= 2 * np.pi * turns + 2 * 2.0 ** -23 * np.abs(want)).all()


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


# ------------------------------------------------------------------ the status word
@pytest.mark.parametrize("call", ["append", "attend", "attend_fp32", "length", "evict", "evict_length"])
def test_a_slot_that_is_not_there_does_not_hide_a_wait_that_ran_out(call):
    P = Pool([40], 8, 1, 64, FP if call == "attend_fp32" else BF, seed=32)
    ctx = B_.Context(64, 1, 1, 64, 4, 64)
    k, out, one = randn((1, 1, 64), P.dt, 1), torch.zeros(1, 64, dtype=P.dt, device=DEV), i32([0, 1])
    if "length" in call:
        P.length[0] = 10 ** 6
    else:
        P.table[0] = P.pages

    def bad():
        if call == "append":
            ctx.d3tom_cache_append(P.cache, None, None, k, k, None, None, None, one, 1, 1, None)
        elif "evict" in call:
            ctx.d3tom_cache_evict(P.cache, i32([8]), None, 1, 40, i32([0]))
        else:
            ctx.d3tom_attn_cached(P.cache, k, one, 1, 1, 1, 40, 0.125, B_.WEIGHT_SET, None, out)

    bad()
    assert ctx.device_status() == B_.ERR_INVALID_ARG
    ctx.reset_device_status()
    ctx.selftest_wait_timeout(10 ** 6)
    bad()
    assert ctx.device_status() == B_.ERR_TIMEOUT
    ctx.reset_device_status()
    assert ctx.device_status() == 0


@pytest.mark.parametrize("dt,H,block", [(BF, 2, 1), (BF, 2, 50), (FP, 2, 1), (FP, 2, 9), (BF, 2, 0)])
def test_a_page_that_is_not_there_is_reported_by_every_kernel(dt, H, block):
    # among several that are, at lengths that fit; where nobody looks, by the weights alone
    P = Pool([300], 16, 1, 128, dt, seed=33)
    P.table[0, 7] = -1
    total = max(1, block)
    q, out = randn((total, H, 128), dt, 1), torch.zeros(total, H * 128, dtype=dt, device=DEV)
    ctx = B_.Context(64, 1, H, 128, 64, 300)
    for mode in (B_.WEIGHT_NONE, B_.WEIGHT_SET)[0 if block else 1:]:
        ctx.d3tom_attn_cached(P.cache, q, i32([0, block]), 1, block, block, 300, 0.1, mode, None, out)
        assert ctx.device_status() == B_.ERR_INVALID_ARG
        ctx.reset_device_status()


# ------------------------------------------------------------------ calls without rows
@pytest.mark.parametrize("dt", [BF, FP])
def test_steps_in_which_nobody_has_rows(dt):
    # tensors of no rows have no address
    C = PagedCache(2, 4, 2, 64, dt, pages=4, page_size=8, max_rows=16, max_length=16, max_scored_rows=4)
    k = randn((5, 2, 64), dt, 1)
    C.append([2, 3], k, k, i32(np.arange(5)), first_weight=torch.tensor([1.0, float("inf"), 2.0, 3.0, 4.0], device=DEV))
    q, kv, none = torch.empty(0, 4, 64, dtype=dt, device=DEV), torch.empty(0, 2, 64, dtype=dt, device=DEV), i32([])
    before = [t.clone() for t in (C.k, C.v, C.weight, C.token)]
    spec = B_.RopeSpec([8, 8])
    C.append([0, 0], kv, kv, none, q=q, q_out=torch.empty_like(q), spec=spec, positions=none.view(0, 2), first_weight=torch.empty(0, device=DEV))
    C.attend([0, 0], q, torch.empty(0, 256, dtype=dt, device=DEV))
    C.ctx.d3tom_rope(spec, q, kv, none.view(0, 2), 0, 2, torch.empty_like(q), torch.empty_like(kv))
    assert C.lengths_h == [2, 3] and C.ctx.device_status() == 0
    for x, y in zip((C.k, C.v, C.weight, C.token), before):
        assert torch.equal(x, y)
    C.attend([0, 0], q, torch.empty(0, 256, dtype=dt, device=DEV), B_.WEIGHT_SET, row_weight=torch.empty(0, device=DEV))
    at = [torch.as_tensor(co.places(C.table_h[b], C.lengths_h[b], 8), device=DEV) for b in range(2)]
    assert C.weight.view(-1)[at[0]].tolist() == [0.0, float("inf")] and C.weight.view(-1)[at[1]].tolist() == [0.0] * 3


# ------------------------------------------------------------------ requests without slots
@pytest.mark.parametrize("dt,H,dh,reference", [(BF, 32, 128, False), (BF, 6, 64, False), (BF, 3, 12, True), (FP, 5, 36, False), (FP, 1, 4, False)])
def test_rows_of_requests_without_slots_are_zero(dt, H, dh, reference):
    # more of them than a warp has lanes, some of one row; what lies behind the last row is left alone
    lens = [0 if b % 3 else 20 for b in range(70)]
    lens[69] = 0
    rows = [b % 4 if b < 69 else 40 for b in range(70)]
    out, _ = check_attention(Pool(lens, 8, 1, dh, dt, seed=34), H, rows, pad=3, reference=reference)
    for b, n in enumerate(lens):
        if n == 0:
            assert not out[cu(rows)[b] : cu(rows)[b + 1]].any()


# ------------------------------------------------------------------ tile widths
@pytest.mark.parametrize("mode", [B_.WEIGHT_NONE, B_.WEIGHT_ADD, B_.WEIGHT_SET])
@pytest.mark.parametrize("H,kv,dh,block", [(3, 1, 64, 11), (2, 2, 64, 33), (8, 2, 64, 16), (5, 5, 64, 64), (3, 1, 128, 11), (4, 4, 128, 64), (2, 1, 128, 20)])
def test_blocks_of_33_to_64_columns(H, kv, dh, block, mode):
    rows = [block, 0, 1, block - 1, block, 2, 0, block]
    P = Pool([0, 1, 127, 128, 129, 640, 33, 1300], 8, kv, dh, BF, seed=35)
    check_attention(P, H, rows, mode, np.random.default_rng(2).uniform(-1, 2, sum(rows)))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("block", [4, 8, 12, 16, 25, 32, 45])
def test_scores_that_grow_along_the_cache_at_every_tile_width(dh, block):
    # 16 .. 180 columns: the running maximum outgrows its reference from tile to tile in one request and falls in the other
    P = Pool([1500, 700], 16, 1, dh, BF, seed=36)
    for b in range(2):
        idx = torch.as_tensor(P.at[b], device=DEV)
        ramp = torch.linspace(0.01, 6.0, 1500, device=DEV) if b == 0 else torch.linspace(5.0, 0.0, 700, device=DEV)
        k = P.flat()[0]
        k[idx] = (k[idx].float() * ramp[:, None, None]).to(BF)
    check_attention(P, 4, [block, 3], B_.WEIGHT_SET, q=randn((block + 5, 4, dh), BF, 3, 3.0))


@pytest.mark.parametrize("dt,dh", [(BF, 128), (BF, 64), (FP, 64)])
@pytest.mark.parametrize("said", [0, 1, 9])
def test_more_rows_than_the_call_was_told(dt, dh, said):
    # max_rows chooses a tile's width, and no result but the order of sums
    lens, rows = [300, 150], [40, 7]
    P = Pool(lens, 16, 2, dh, dt, seed=37)
    q, ctx = randn((47, 4, dh), dt, 1), B_.Context(64, 2, 4, dh, 47, 300)
    res = []
    for most in (40, said):
        w = torch.zeros_like(P.weight)
        out = torch.zeros(47, 4 * dh, dtype=dt, device=DEV)
        cache = B_.Cache(P.k, P.v, w, P.token, P.table, P.length)
        ctx.d3tom_attn_cached(cache, q, i32(cu(rows)), 2, 47, most, 300, dh ** -0.5, B_.WEIGHT_SET, None, out)
        res.append((f64(out), f64(w)))
    # bf16: two roundings of P and one of the result on either side, of sums of |v| p up to 4
    assert np.abs(res[0][0] - res[1][0]).max() <= (4 * 4 * 2.0 ** -8 if dt == BF else 1e-4)
    assert np.abs(res[0][1] - res[1][1]).max() <= 1e-3 * np.abs(res[0][1]).max() and ctx.device_status() == 0


# ------------------------------------------------------------------ slots that are not there
@pytest.mark.parametrize("dt,H,kv,dh,block", [(BF, 2, 2, 128, 1), (BF, 2, 2, 128, 32), (BF, 2, 2, 128, 40), (BF, 4, 1, 128, 30), (BF, 2, 2, 64, 20), (BF, 2, 1, 64, 40),
                                              (FP, 4, 2, 64, 1), (FP, 4, 2, 64, 9)])
@pytest.mark.parametrize("mode", [B_.WEIGHT_ADD, B_.WEIGHT_SET])
def test_weights_of_slots_that_are_not_there_keep_every_bit(dt, H, kv, dh, block, mode):
    P = Pool([700, 90], 16, kv, dh, dt, seed=38)
    P.table[0, 3] = P.pages
    P.length[1] = 10 ** 6                        # behind max_length: 90 slots are looked at
    P.table[1, 6:] = -1
    gone, whole = P.at[0][48:64], P.at[0]
    there = [np.concatenate([whole[:48], whole[64:]]), P.at[1]]
    q, rows = randn((block + 1, H, dh), dt, 1), [block, 1]
    before = P.copy()
    out = torch.zeros(block + 1, H * dh, dtype=dt, device=DEV)
    ctx = B_.Context(64, 2, H, dh, block + 1, 700)
    ctx.d3tom_attn_cached(P.cache, q, i32(cu(rows)), 2, block + 1, block, 700, dh ** -0.5, mode, None, out)
    assert ctx.device_status() == B_.ERR_INVALID_ARG
    k1, v1, w1, t1 = P.flat()
    for b in range(2):
        lo, hi, idx = cu(rows)[b], cu(rows)[b + 1], torch.as_tensor(there[b], device=DEV)
        if b == 1:                               # its table ends with the page of slot 95: the slots behind its 90 are anything
            continue
        o, p, mag, _ = co.attend(f64(q[lo:hi]), f64(k1[idx]), f64(v1[idx]), dh ** -0.5)
        assert (np.abs(f64(out[lo:hi]).reshape(o.shape) - o) <= 2.0 ** -7 * mag + 1e-4).all()
        want = p.sum(axis=(0, 1)) + (f64(before[2])[there[b]] if mode == B_.WEIGHT_ADD else 0.0)
        assert (np.abs(f64(w1)[there[b]] - want) <= 5e-4 * want).all()
    touched = np.zeros(len(w1), bool)
    touched[there[0]] = True
    touched[co.places(P.table_h[1], 96, 16)] = True
    assert not touched[gone].any()
    rest = torch.as_tensor(~touched, device=DEV)
    assert torch.equal(w1[rest], before[2][rest]) and torch.equal(t1, before[3])
    assert torch.equal(k1.nan_to_num(99), before[0].nan_to_num(99)) and torch.equal(v1.nan_to_num(99), before[1].nan_to_num(99))


# ------------------------------------------------------------------ a merged prefix, cached and decoded against
@pytest.mark.parametrize("dt,H,dh,page", [(BF, 4, 128, 16), (BF, 4, 64, 24), (FP, 3, 32, 5)])
def test_a_merged_prefix_goes_into_the_pages_and_is_attended_to(dt, H, dh, page):
    """d3tom_merge_kv's shortened K and V with their source rows as token numbers -> PagedCache -> a response block with weights ->
    eviction that keeps the prompt; against fp64 on the merged rows that the merge itself is checked to give."""
    n_vis, n_prompt, keep = [150, 61], [9, 4], [40, 20]
    lens, out_lens = [v + p for v, p in zip(n_vis, n_prompt)], [k + p for k, p in zip(keep, n_prompt)]
    D, total, total_out = H * dh, sum(lens), sum(out_lens)
    rng = np.random.default_rng(5)
    kept = [np.sort(rng.choice(v, k, replace=False)).astype(np.int32) for v, k in zip(n_vis, keep)]
    k, v = randn((total, D), dt, 1), randn((total, D), dt, 2)
    k_out, v_out = torch.empty(total_out, D, dtype=dt, device=DEV), torch.empty(total_out, D, dtype=dt, device=DEV)
    assign, count, src = i32(np.zeros(sum(n_vis))), i32(np.zeros(sum(keep))), i32(np.zeros(total_out))
    merge = B_.Context(total, 2, H, dh, 1, max(n_vis))
    merge.d3tom_merge_kv(B_.AGG_MEAN, k, v, i32(cu(lens)), i32(n_vis), i32(cu(n_vis)), i32(np.concatenate(kept)), i32(cu(keep)), 2, D, total,
                         total_out, max(n_vis), max(keep), k_out, v_out, i32(cu(out_lens)), assign, count, src)
    # prompt rows are copies, and the merge says where every row came from
    src_h = src.cpu().numpy()
    for b in range(2):
        rows_b = np.concatenate([kept[b], np.arange(n_vis[b], lens[b])]) + cu(lens)[b]
        assert np.array_equal(src_h[cu(out_lens)[b] : cu(out_lens)[b + 1]], rows_b)
        prompt = slice(cu(out_lens)[b] + keep[b], cu(out_lens)[b + 1])
        assert torch.equal(k_out[prompt], k[torch.as_tensor(src_h[prompt], device=DEV).long()])
    block = [5, 3]
    C = PagedCache(2, H, H, dh, dt, pages=sum(-(-(n + r) // page) for n, r in zip(out_lens, block)), page_size=page, max_rows=total_out,
                   max_length=max(out_lens) + 5, max_scored_rows=8)
    is_prompt = np.concatenate([np.arange(n) >= q for n, q in zip(out_lens, keep)])
    first = torch.where(torch.as_tensor(is_prompt, device=DEV), float("inf"), 0.0).to(FP)
    C.append(out_lens, k_out, v_out, src, first_weight=first)
    q, kb, vb = randn((8, H, dh), dt, 3), randn((8, H, dh), dt, 4), randn((8, H, dh), dt, 5)
    out = torch.empty(8, D, dtype=dt, device=DEV)
    C.append(block, kb, vb, i32(np.arange(8) + 100000))
    C.attend(block, q, out, B_.WEIGHT_SET)
    mass = []
    for b in range(2):
        lo, hi, n = cu(block)[b], cu(block)[b + 1], out_lens[b]
        at = torch.as_tensor(co.places(C.table_h[b], n + block[b], page), device=DEV)
        part = slice(cu(out_lens)[b], cu(out_lens)[b + 1])
        keys, values = (torch.cat([x[part].view(-1, H, dh), y[lo:hi]]) for x, y in ((k_out, kb), (v_out, vb)))
        assert torch.equal(C.k.view(-1, H, dh)[at], keys) and torch.equal(C.v.view(-1, H, dh)[at], values)
        assert C.token.view(-1)[at].tolist() == src_h[part].tolist() + list(range(100000 + lo, 100000 + hi))
        o, p, mag, _ = co.attend(f64(q[lo:hi]), f64(keys), f64(values), dh ** -0.5)
        # P and the result rounded (bf16), sums of dh products and of up to 54 terms (fp32)
        assert (np.abs(f64(out[lo:hi]).reshape(o.shape) - o) <= (2.0 ** -7 if dt == BF else 0) * mag + 5e-4 * mag).all()
        m = p.sum(axis=(0, 1))
        got = f64(C.weight.view(-1)[at])
        assert np.isinf(got[keep[b] : n]).all() and (np.abs(np.delete(got - m, np.s_[keep[b] : n])) <= 5e-4 * np.delete(m, np.s_[keep[b] : n])).all()
        mass.append(got[:n])
    C.drop_last(block)
    budget = [12, 10]
    want = [[src_h[cu(out_lens)[b] + j] for j in range(out_lens[b])] for b in range(2)]
    for b in range(2):
        n, moves = co.evict(mass[b], None, budget[b])
        for s, d in moves:
            want[b][d] = want[b][s]
        want[b] = want[b][:n]
    C.evict(budget)
    for b in range(2):
        at = torch.as_tensor(co.places(C.table_h[b], C.lengths_h[b], page), device=DEV)
        assert C.token.view(-1)[at].tolist() == want[b]
        assert set(src_h[is_prompt & (np.repeat([0, 1], out_lens) == b)].tolist()) <= set(want[b])
    assert C.ctx.device_status() == 0 and merge.device_status() == 0
