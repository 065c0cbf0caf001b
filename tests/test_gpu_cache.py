"""Rotary positions and the K/V cache in pages against their plain fp64 definitions.

Error bounds.  bf16 results are rounded once (2^-8 of the value).  Rotation: the angle is off by less than 8e-7 with the
roundings of cosine, sine (2 ulp) and three fp32 operations.  Attention: a score is off by at most (dh + 8) 2^-24 sum |q||k| scale,
an exponential by twice 2^-22 more, and a quotient of sums has that twice; n terms summed in fp32 add n 2^-24; on the tensor cores
every probability is rounded to bf16 (2^-8) before the second product."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as co
from paper_2511_12280_b200 import binding as B_
from paper_2511_12280_b200.cache import PagedCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, FP: 2.0 ** -24}


def f64(t):
    return t.detach().double().cpu().numpy()


def i32(a):
    return torch.as_tensor(np.asarray(a, dtype=np.int32), device=DEV)


def cu(a):
    return np.concatenate([[0], np.cumsum(a)]).astype(np.int32)


def randn(shape, dt, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dt).to(DEV)


# ------------------------------------------------------------------ rotary positions
ROPES = [  # dtype, H, kv, dh, sections, neighbours, per axis, theta
    (BF, 4, 2, 128, [16, 24, 24], False, False, 1e4), (BF, 3, 3, 64, [8, 8, 16], True, True, 1e6), (BF, 2, 1, 64, [5, 3, 3], False, True, 1e4),
    (BF, 2, 2, 128, [0, 7, 1], False, False, 100.0), (BF, 2, 1, 64, [3, 2, 4], True, False, 1e4), (FP, 4, 4, 128, [64], False, False, 1e4),
    (FP, 3, 1, 20, [3, 2], False, False, 1e4), (FP, 2, 2, 36, [7, 0, 5], True, True, 1e4), (FP, 5, 5, 4, [1, 1], False, True, 1.0),
]


@pytest.mark.parametrize("dt,H,kv,dh,sec,nb,per,theta", ROPES)
@pytest.mark.parametrize("rows", [1, 7, 130])
def test_rope(dt, H, kv, dh, sec, nb, per, theta, rows):
    ctx = B_.Context(256, 1, H, dh, 1, 1)
    spec = B_.RopeSpec(sec, theta, B_.PAIR_NEIGHBOURS if nb else B_.PAIR_HALVES, B_.LADDER_PER_AXIS if per else B_.LADDER_SHARED)
    rng = np.random.default_rng(rows)
    pos = rng.integers(-2 ** 31, 2 ** 31, (rows, len(sec)))
    pos[: rows // 2] = rng.integers(0, 5000, (rows // 2, len(sec)))
    q, k = randn((rows, H, dh), dt, 1), randn((rows, kv, dh), dt, 2)
    ang = co.rope_angles(pos, sec, theta, per)
    for inverse in (False, True):
        q_out, k_out = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
        ctx.d3tom_rope(spec, q, k, i32(pos), rows, kv, q_out, k_out, inverse=inverse)
        for x, y in ((q, q_out), (k, k_out)):
            want, size = co.rope(f64(x), ang, nb, inverse), np.abs(f64(x)).max()
            assert (np.abs(f64(y) - want) <= HALF[dt] * np.abs(want) + 2e-6 * size).all()
            n = 2 * sum(sec)
            assert torch.equal(y[..., n:], x[..., n:])              # numbers that do not turn are copies
        a, b = q.clone(), k.clone()
        ctx.d3tom_rope(spec, a, b, i32(pos), rows, kv, a, b, inverse=inverse)     # in place
        assert torch.equal(a, q_out) and torch.equal(b, k_out)
        only = torch.zeros_like(q)
        ctx.d3tom_rope(spec, q, None, i32(pos), rows, 0, only, None, inverse=inverse)
        assert torch.equal(only, q_out)
    assert ctx.device_status() == 0


def test_rope_inverse_is_its_gradient():
    # <R x, g> = <x, R^-1 g>, and the same from differences of R
    H, dh, rows = 3, 64, 5
    ctx, spec = B_.Context(64, 1, H, dh, 1, 1), B_.RopeSpec([8, 8, 8])
    x, g, pos = randn((rows, H, dh), FP, 3), randn((rows, H, dh), FP, 4), i32(np.arange(15).reshape(5, 3) * 1001)
    y, back = torch.empty_like(x), torch.empty_like(x)
    ctx.d3tom_rope(spec, x, None, pos, rows, 0, y, None)
    ctx.d3tom_rope(spec, g, None, pos, rows, 0, back, None, inverse=True)
    gx, gb = f64(x), f64(back)
    assert abs((f64(y) * f64(g)).sum() - (gx * gb).sum()) <= 1e-5 * np.sqrt((gx ** 2).sum() * (gb ** 2).sum())
    step = 0.5
    for at in ((0, 0, 0), (2, 1, 40), (4, 2, 63), (3, 0, 24)):
        two = []
        for sign in (1, -1):
            z = x.clone()
            z[at] += sign * step
            ctx.d3tom_rope(spec, z, None, pos, rows, 0, y, None)
            two.append((f64(y) * f64(g)).sum())
        assert abs((two[0] - two[1]) / (2 * step) - gb[at]) <= 1e-4


def test_rope_position_zero_copies_and_rows_end():
    ctx, spec = B_.Context(64, 1, 2, 64, 1, 1), B_.RopeSpec([32])
    q = randn((6, 2, 64), BF, 5)
    out = torch.full_like(q, 7.0)
    ctx.d3tom_rope(spec, q, None, i32(np.zeros((6, 1))), 4, 0, out, None)
    assert torch.equal(out[:4], q[:4]) and (out[4:] == 7).all()


# ------------------------------------------------------------------ a cache to test with
class Pool:
    def __init__(self, lens, page, kv, dh, dt, seed=0, extra=3, width=0, fill=1.0):
        rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in lens]
        self.pages = sum(need) + extra
        order = rng.permutation(self.pages).astype(np.int32)
        self.table_h = np.full((len(lens), max(1, max(need)) + width), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table_h[b, :n] = order[at : at + n]
            at += n
        self.lens, self.page, self.kv, self.dh, self.dt = list(lens), page, kv, dh, dt
        self.k = torch.full((self.pages, page, kv, dh), float("nan"), dtype=dt, device=DEV)    # what no request has is NaN
        self.v = torch.full_like(self.k, float("nan"))
        self.weight = torch.full((self.pages, page), -5.0, device=DEV)
        self.token = torch.full((self.pages, page), -5, dtype=torch.int32, device=DEV)
        self.table, self.length = i32(self.table_h), i32(lens)
        self.at = [co.places(self.table_h[b], n, page) for b, n in enumerate(lens)]
        for b, n in enumerate(lens):
            idx = torch.as_tensor(self.at[b], device=DEV)
            self.k.view(-1, kv, dh)[idx] = randn((n, kv, dh), dt, seed * 100 + 2 * b + 1, fill)
            self.v.view(-1, kv, dh)[idx] = randn((n, kv, dh), dt, seed * 100 + 2 * b + 2)
            self.weight.view(-1)[idx] = torch.rand(n, generator=torch.Generator().manual_seed(b)).to(DEV)
            self.token.view(-1)[idx] = torch.arange(n, dtype=torch.int32, device=DEV)
        self.cache = B_.Cache(self.k, self.v, self.weight, self.token, self.table, self.length)

    def flat(self):
        return (self.k.view(-1, self.kv, self.dh), self.v.view(-1, self.kv, self.dh), self.weight.view(-1), self.token.view(-1))

    def copy(self):
        return [t.clone() for t in self.flat()]


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dt,H,kv,dh,page", [(BF, 4, 2, 128, 16), (BF, 3, 3, 64, 24), (FP, 4, 1, 36, 5), (FP, 2, 2, 64, 1)])
@pytest.mark.parametrize("turn", [True, False])
def test_append(dt, H, kv, dh, page, turn):
    lens, rows = [40, 3, 0, 17, 1], [7, 3, 0, 0, 1]
    P = Pool(lens, page, kv, dh, dt, seed=1)
    total, sec = sum(rows), [4, 5, 3]
    spec = B_.RopeSpec(sec, 1e4) if turn else None
    ctx = B_.Context(64, 5, H, dh, 1, 1)
    pos = np.random.default_rng(0).integers(0, 2 ** 20, (total + 2, 3))
    q, k, v = randn((total + 2, H, dh), dt, 11), randn((total + 2, kv, dh), dt, 12), randn((total + 2, kv, dh), dt, 13)
    tokens, first = i32(np.arange(total + 2) + 500), torch.arange(total + 2, dtype=FP, device=DEV) + 0.5
    first[2] = float("inf")
    q_out = torch.full_like(q, 3.0)
    before = P.copy()
    ctx.d3tom_cache_append(P.cache, spec, q, k, v, i32(pos) if turn else None, tokens, first, i32(cu(rows)), 5, total + 2, q_out)
    assert ctx.device_status() == 0
    ang = co.rope_angles(pos, sec, 1e4, False)
    kr, qr = (co.rope(f64(k), ang), co.rope(f64(q), ang)) if turn else (f64(k), f64(q))
    assert (np.abs(f64(q_out[:total]) - qr[:total]) <= (HALF[dt] * np.abs(qr[:total]) + 2e-5 if turn else 0)).all()
    assert (q_out[total:] == 3).all()                               # rows behind the last request
    k1, v1, w1, t1 = P.flat()
    touched = np.zeros(len(w1), bool)
    for b, (n, r) in enumerate(zip(lens, rows)):
        dst, src = P.at[b][n - r :], np.arange(cu(rows)[b], cu(rows)[b + 1])
        touched[dst] = True
        assert (np.abs(f64(k1)[dst] - kr[src]) <= (HALF[dt] * np.abs(kr[src]) + 2e-5 if turn else 0)).all()
        assert np.array_equal(f64(v1)[dst], f64(v)[src])
        assert np.array_equal(f64(w1)[dst], f64(first)[src]) and np.array_equal(t1.cpu().numpy()[dst], src + 500)
    rest = torch.as_tensor(~touched, device=DEV)
    for x, y in zip(P.flat(), before):
        assert torch.equal(x[rest].nan_to_num(99), y[rest].nan_to_num(99))


def test_append_without_queries_tokens_and_weights():
    P = Pool([5], 8, 2, 64, BF, seed=2)
    k, v = randn((2, 2, 64), BF, 1), randn((2, 2, 64), BF, 2)
    B = B_.Cache(P.k, P.v, P.weight, None, P.table, P.length)
    ctx = B_.Context(8, 1, 2, 64, 1, 1)
    ctx.d3tom_cache_append(B, None, None, k, v, None, None, None, i32([0, 2]), 1, 2, None)
    k1, v1, w1, t1 = P.flat()
    at = torch.as_tensor(P.at[0], device=DEV)
    assert torch.equal(k1[at[3:]], k) and torch.equal(v1[at[3:]], v) and (w1[at[3:]] == 0).all()
    assert t1[at].tolist() == [0, 1, 2, 3, 4]


def test_append_drops_rows_without_a_slot():
    P = Pool([5, 9], 8, 1, 64, FP, seed=3)
    P.table[1, 1] = P.pages                                          # not a page of the pool
    P.length[0] = 1                                                  # two new rows, one slot
    before = P.copy()
    k = randn((4, 1, 64), FP, 1)
    ctx = B_.Context(8, 2, 1, 64, 1, 1)
    ctx.d3tom_cache_append(P.cache, None, None, k, k, None, i32([70, 71, 72, 73]), None, i32([0, 2, 4]), 2, 4, None)
    assert ctx.device_status() == B_.ERR_INVALID_ARG
    ctx.reset_device_status()
    k1, _, _, t1 = P.flat()
    put = {int(P.at[0][0]): 1, int(P.at[1][7]): 2}
    for j in range(len(t1)):
        want = k[put[j]] if j in put else before[0][j]
        assert torch.equal(k1[j].nan_to_num(99), want.nan_to_num(99)) and int(t1[j]) == (70 + put[j] if j in put else int(before[3][j]))


# ------------------------------------------------------------------ attention
def check_attention(P, H, rows, mode=B_.WEIGHT_NONE, factors=None, pad=2, seed=5, ctx=None, q=None, reference=False, stream=None):
    dt, dh, B = P.dt, P.dh, len(P.lens)
    total = sum(rows)
    ctx = ctx or B_.Context(max(1, total + pad), B, H, dh, max(1, total + pad), max(1, max(P.lens)))
    if reference:
        ctx.set_reference_kernels(True)
    q = randn((total + pad, H, dh), dt, seed) if q is None else q
    out = torch.full((total + pad, H * dh), 3.0, dtype=dt, device=DEV)
    f = None if factors is None else torch.as_tensor(np.concatenate([factors, np.full(pad, 1e9)]), dtype=FP, device=DEV)
    before = P.copy()
    scale = 1.0 / np.sqrt(dh)
    args = (P.cache, q, i32(cu(rows)), B, total + pad, max(rows) if rows else 0, max(P.lens), scale, mode, f, out)
    ctx.d3tom_attn_cached(*args)
    assert ctx.device_status() == 0
    assert (out[total:] == 3).all()
    k1, v1, w1, _ = P.flat()
    assert torch.equal(k1.nan_to_num(99), before[0].nan_to_num(99)) and torch.equal(v1.nan_to_num(99), before[1].nan_to_num(99))
    tensor = dt == BF and not reference
    w_want, touched = f64(before[2]), np.zeros(len(w1), bool)
    for b, n in enumerate(P.lens):
        lo, hi = cu(rows)[b], cu(rows)[b + 1]
        idx = torch.as_tensor(P.at[b], device=DEV)
        o, p, mag, reach = co.attend(f64(q[lo:hi]), f64(k1[idx]), f64(v1[idx]), float(np.float32(scale)))
        delta = 2 * ((dh + 8) * 2.0 ** -24 * reach + 2.0 ** -21) + n * 2.0 ** -24
        got = f64(out[lo:hi]).reshape(o.shape)
        assert np.isfinite(got).all()
        err, tol = np.abs(got - o), HALF[dt] * np.abs(o) + ((2.0 ** -8 if tensor else 0) + delta) * mag
        assert (err <= tol).all(), (b, n, float((err / np.maximum(tol, 1e-30)).max()))
        if mode != B_.WEIGHT_NONE:
            g = np.ones(hi - lo) if factors is None else factors[lo:hi].astype(np.float32).astype(np.float64)
            mass = np.einsum("rhn,r->n", p, g)
            had = w_want[P.at[b]] if mode == B_.WEIGHT_ADD else 0.0
            w_got = f64(w1)[P.at[b]]
            tol = (delta + (H * (hi - lo) + 8) * 2.0 ** -24) * np.einsum("rhn,r->n", p, np.abs(g)) + 2.0 ** -23 * np.abs(had) + 1e-35
            assert (np.abs(w_got - (mass + had)) <= tol).all(), (b, n)
            touched[P.at[b]] = True
    keep = torch.as_tensor(~touched, device=DEV)
    assert torch.equal(w1[keep], before[2][keep])
    # again: the same bits
    again = torch.full_like(out, 3.0)
    w_first = w1.clone()
    w1.copy_(before[2])
    ctx.d3tom_attn_cached(*args[:-1], again)
    assert torch.equal(again, out) and torch.equal(w1, w_first)
    return out, ctx


LENS = [0, 1, 127, 128, 129, 640, 33, 1300]


@pytest.mark.parametrize("dt,page", [(BF, 16), (BF, 8), (BF, 48), (BF, 128), (BF, 264), (FP, 16), (FP, 7)])
@pytest.mark.parametrize("H,kv,dh", [(4, 4, 128), (8, 2, 64)])
def test_attention_one_token_of_each_request(dt, page, H, kv, dh):
    P = Pool(LENS, page, kv, dh, dt, seed=4)
    check_attention(P, H, [1] * len(LENS), B_.WEIGHT_ADD)


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("H,kv,dh", [(2, 2, 128), (7, 1, 64), (6, 3, 128), (16, 2, 64)])
@pytest.mark.parametrize("block", [3, 17, 40])
def test_attention_blocks(dt, H, kv, dh, block):
    # 3 .. 320 rows x query heads per key head: every tile width, several tiles, tiles that are not full
    rows = [block, 0, 1, block - 1, block, 2, 0, block]
    P = Pool(LENS, 16, kv, dh, dt, seed=6)
    factors = np.random.default_rng(1).uniform(-1, 2, sum(rows))
    check_attention(P, H, rows, B_.WEIGHT_SET, factors)


@pytest.mark.parametrize("dt,dh,H,kv", [(BF, 128, 4, 4), (BF, 64, 32, 1), (FP, 20, 3, 1), (FP, 128, 2, 1)])
def test_attention_over_one_long_request(dt, dh, H, kv):
    # one request over all SMs: every CTA has a part of an item
    check_attention(Pool([30011], 16, kv, dh, dt, seed=7, extra=0), H, [1], B_.WEIGHT_SET, pad=0)


@pytest.mark.parametrize("dt,dh", [(BF, 128), (BF, 64), (FP, 64), (FP, 4)])
def test_attention_of_more_requests_than_lanes(dt, dh):
    lens = [(37 * b) % 301 for b in range(70)]
    rows = [b % 3 for b in range(70)]
    check_attention(Pool(lens, 8, 1, dh, dt, seed=8), 2, rows, B_.WEIGHT_ADD, pad=0)


@pytest.mark.parametrize("dh", [64, 128, 40])
def test_bf16_attention_on_the_plain_kernels(dh):
    check_attention(Pool(LENS, 12, 2, dh, BF, seed=9), 6, [2] * len(LENS), B_.WEIGHT_ADD, reference=True)


@pytest.mark.parametrize("dt,dh", [(BF, 128), (BF, 64), (FP, 64)])
def test_attention_with_scores_that_grow_along_the_cache(dt, dh):
    # the running maximum rises by far more than 2^8 from tile to tile, and falls; rows differ
    P = Pool([1500, 700], 16, 1, dh, dt, seed=10)
    for b in range(2):
        idx = torch.as_tensor(P.at[b], device=DEV)
        n = len(P.at[b])
        ramp = torch.linspace(0.01, 6.0, n, device=DEV) if b == 0 else torch.linspace(5.0, 0.0, n, device=DEV)
        k = P.flat()[0]
        k[idx] = (k[idx].float() * ramp[:, None, None]).to(dt)
    check_attention(P, 4, [5, 2], B_.WEIGHT_SET, q=randn((9, 4, dh), dt, 3, 3.0))


@pytest.mark.parametrize("mode", [B_.WEIGHT_NONE, B_.WEIGHT_SET])
def test_attention_of_a_token_with_more_heads_per_key_head_than_a_tile_has_columns(mode):
    check_attention(Pool([333, 90], 16, 1, 64, BF, seed=24), 144, [1, 2], mode)
    check_attention(Pool([333, 90], 16, 1, 64, FP, seed=24), 144, [1, 2], mode)


def test_two_streams_read_one_cache_at_once():
    lens = [900, 30, 2000, 411]
    P = Pool(lens, 16, 2, 64, BF, seed=25)
    runs = []
    for rows in ([1] * 4, [40] * 4, [3, 0, 17, 1]):
        total = sum(rows)
        ctx = B_.Context(total, 4, 8, 64, 1, 1)
        q = randn((total, 8, 64), BF, total)
        out = torch.zeros(total, 512, dtype=BF, device=DEV)
        args = (P.cache, q, i32(cu(rows)), 4, total, max(rows), 2000, 0.125, B_.WEIGHT_NONE, None)
        ctx.d3tom_attn_cached(*args, out)
        runs.append((ctx, args, out, [torch.zeros_like(out) for _ in range(20)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(20):
        for ctx, args, _, outs, stream in runs:
            ctx.d3tom_attn_cached(*args, outs[i], stream=stream)
    torch.cuda.synchronize()
    for ctx, _, out, outs, _ in runs:
        assert ctx.device_status() == 0 and all(torch.equal(out, x) for x in outs)


@pytest.mark.parametrize("dt", [BF, FP])
def test_attention_of_equal_keys_is_the_mean(dt):
    n, dh = 1000, 64
    P = Pool([n], 8, 1, dh, dt, seed=11)
    idx = torch.as_tensor(P.at[0], device=DEV)
    P.flat()[0][idx] = 1.0
    out, _ = check_attention(P, 1, [1], B_.WEIGHT_SET)
    mean = f64(P.flat()[1][idx]).mean(axis=0).ravel()
    assert np.abs(f64(out[0]) - mean).max() <= 2.0 ** -8 * np.abs(mean).max() + 2.0 ** -8
    assert np.abs(f64(P.flat()[2][idx]) - 1.0 / n).max() <= 1e-5 / n * 10


@pytest.mark.parametrize("dt", [BF, FP])
def test_attention_without_rows_or_slots(dt):
    P = Pool([0, 0, 0], 8, 2, 64, dt, seed=12, width=1)
    check_attention(P, 4, [1, 0, 3], B_.WEIGHT_SET)
    P = Pool([300, 20], 8, 2, 64, dt, seed=12)
    check_attention(P, 4, [0, 0], B_.WEIGHT_SET)                     # nobody looks: the weights are 0
    check_attention(P, 4, [0, 0], B_.WEIGHT_ADD)


@pytest.mark.parametrize("dt", [BF, FP])
def test_attention_of_no_rows_at_all(dt):
    P = Pool([300, 20], 8, 2, 64, dt, seed=12)
    q = randn((1, 4, 64), dt, 1)
    out = torch.full((1, 256), 3.0, dtype=dt, device=DEV)
    ctx = B_.Context(4, 2, 4, 64, 4, 300)
    before = P.copy()[2]
    for mode, want in ((B_.WEIGHT_NONE, None), (B_.WEIGHT_ADD, None), (B_.WEIGHT_SET, 0.0)):
        ctx.d3tom_attn_cached(P.cache, q, i32([0, 0, 0]), 2, 0, 0, 300, 0.125, mode, None, out)
        for b in range(2):
            at = torch.as_tensor(P.at[b], device=DEV)
            assert torch.equal(P.flat()[2][at], before[at] if want is None else torch.zeros_like(before[at]))
    assert (out == 3).all() and ctx.device_status() == 0


@pytest.mark.parametrize("block,H,kv", [(32, 2, 2), (70, 4, 1), (9, 8, 2)])
def test_weights_leave_out_a_page_that_is_not_there(block, H, kv):
    # the same with so many rows that the weights come from a second pass over the keys
    P = Pool([700], 16, kv, 128, BF, seed=23)
    P.table[0, 3] = P.pages
    whole = P.at[0]
    there = np.concatenate([whole[:48], whole[64:]])
    q = randn((block, H, 128), BF, 1)
    out = torch.zeros(block, H * 128, dtype=BF, device=DEV)
    ctx = B_.Context(block, 1, H, 128, block, 700)
    ctx.d3tom_attn_cached(P.cache, q, i32([0, block]), 1, block, block, 700, 128 ** -0.5, B_.WEIGHT_SET, None, out)
    assert ctx.device_status() == B_.ERR_INVALID_ARG
    k1, v1, w1, _ = P.flat()
    idx = torch.as_tensor(there, device=DEV)
    o, p, mag, _ = co.attend(f64(q), f64(k1[idx]), f64(v1[idx]), 128 ** -0.5)
    assert (np.abs(f64(out).reshape(o.shape) - o) <= 2.0 ** -7 * mag + 1e-4).all()
    mass = p.sum(axis=(0, 1))
    assert (np.abs(f64(w1)[there] - mass) <= 1e-3 * mass).all()
    gone = torch.as_tensor(whole[48:64], device=DEV)
    assert torch.equal(w1[gone], P.copy()[2][gone]) and torch.isfinite(w1[gone]).all()


@pytest.mark.parametrize("dt", [BF, FP])
def test_attention_leaves_out_what_is_not_there(dt):
    # a page that is not in the pool, and a length beyond the table: as if those slots were not there
    P = Pool([300, 64], 16, 1, 64, dt, seed=13)
    P.table[0, 4] = -7
    P.length[1] = 10 ** 6
    whole = P.at[0]
    P.at[0] = np.concatenate([whole[:64], whole[80:]])
    P.lens = [284, 64]
    ctx, H = B_.Context(8, 2, 2, 64, 8, 300), 2
    q = randn((3, H, 64), dt, 1)
    out = torch.zeros(3, H * 64, dtype=dt, device=DEV)
    P.table[1, 4:] = -1
    ctx.d3tom_attn_cached(P.cache, q, i32([0, 2, 3]), 2, 3, 2, 300, 0.125, B_.WEIGHT_SET, None, out)
    assert ctx.device_status() == B_.ERR_INVALID_ARG
    ctx.reset_device_status()
    assert ctx.device_status() == 0
    k1, v1, w1, _ = P.flat()
    for b, (lo, hi) in enumerate(((0, 2), (2, 3))):
        idx = torch.as_tensor(P.at[b], device=DEV)
        o, p, mag, _ = co.attend(f64(q[lo:hi]), f64(k1[idx]), f64(v1[idx]), 0.125)
        got = f64(out[lo:hi]).reshape(o.shape)
        assert (np.abs(got - o) <= 2.0 ** -7 * mag + 1e-4).all()
        assert np.abs(f64(w1)[P.at[b]] - p.sum(axis=(0, 1))).max() <= 1e-4
    assert (w1[torch.as_tensor(whole[64:80], device=DEV)] != w1[torch.as_tensor(whole[:1], device=DEV)]).any()


def test_attention_with_infinite_and_nan_keys_of_other_requests():
    P = Pool([200, 77], 16, 2, 64, BF, seed=14)
    idx = torch.as_tensor(P.at[1], device=DEV)
    P.flat()[0][idx], P.flat()[1][idx] = float("inf"), float("nan")
    ctx = B_.Context(4, 2, 2, 64, 4, 200)
    q, out = randn((2, 2, 64), BF, 1), torch.zeros(2, 128, dtype=BF, device=DEV)
    ctx.d3tom_attn_cached(P.cache, q, i32([0, 1, 2]), 2, 2, 1, 200, 0.125, B_.WEIGHT_NONE, None, out)
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all()


def test_attention_beyond_32_bit_offsets():
    # pools of more than 2^32 numbers each; the request's pages lie at their end
    page, kv, dh = 128, 8, 128
    pages = 2 ** 32 // (page * kv * dh) + 24
    if torch.cuda.mem_get_info()[0] < 3 * pages * page * kv * dh * 2:
        pytest.skip("not enough memory")
    k = torch.empty(pages, page, kv, dh, dtype=BF, device=DEV)
    v = torch.empty_like(k)
    lens = [1200, 700]
    table = np.arange(pages - 1, pages - 1 - 20, -1, dtype=np.int32).reshape(2, 10)
    P = Pool([1, 1], page, kv, dh, BF)
    P.k, P.v, P.pages, P.lens, P.table_h = k, v, pages, lens, table
    P.weight, P.token = torch.zeros(pages, page, device=DEV), torch.zeros(pages, page, dtype=torch.int32, device=DEV)
    P.table, P.length, P.at = i32(table), i32(lens), [co.places(table[b], n, page) for b, n in enumerate(lens)]
    P.cache = B_.Cache(k, v, P.weight, P.token, P.table, P.length)
    ctx = B_.Context(4096, 2, 16, dh, 8, 1200)
    spec = B_.RopeSpec([64])
    rows = randn((sum(lens), kv, dh), BF, 1)
    tok = i32(np.concatenate([np.arange(n) for n in lens]))
    ctx.d3tom_cache_append(P.cache, None, None, rows, rows, None, tok, None, i32(cu(lens)), 2, sum(lens), None)
    q = randn((2, 16, dh), BF, 2)
    for dt_ref in (False, True):
        ctx.set_reference_kernels(dt_ref)
        out = torch.zeros(2, 16 * dh, dtype=BF, device=DEV)
        ctx.d3tom_attn_cached(P.cache, q, i32([0, 1, 2]), 2, 2, 1, 1200, dh ** -0.5, B_.WEIGHT_SET, None, out)
        for b in range(2):
            x = f64(rows[cu(lens)[b] : cu(lens)[b + 1]])
            o, p, mag, _ = co.attend(f64(q[b : b + 1]), x, x, dh ** -0.5)
            assert (np.abs(f64(out[b]) - o.ravel()) <= 2.0 ** -7 * mag.ravel() + 1e-4).all()
    ctx.d3tom_cache_evict(P.cache, i32([100, 650]), None, 2, 1200, P.length)
    assert P.length.tolist() == [100, 650] and ctx.device_status() == 0
    for b, n in enumerate([100, 650]):
        at = torch.as_tensor(P.at[b][:n], device=DEV)
        t = P.token.view(-1)[at].long() + int(cu(lens)[b])
        assert torch.equal(k.view(-1, kv, dh)[at], rows[t]) and torch.equal(v.view(-1, kv, dh)[at], rows[t])


# ------------------------------------------------------------------ eviction
def check_evict(P, budget, protect=None, in_place=True, max_length=None):
    B, before = len(P.lens), P.copy()
    need = B * ((max_length or max(P.lens)) + 1)
    H = P.kv
    ctx = B_.Context(max(1, -(-need // (H * P.dh))), B, H, P.dh, 1, 1)     # not a word more than it asks for
    length_out = P.length if in_place else i32([-3] * B)
    ctx.d3tom_cache_evict(P.cache, i32(budget), None if protect is None else i32(protect), B, max_length or max(P.lens), length_out)
    assert ctx.device_status() == 0
    want = [t.clone() for t in before]
    lens = []
    w, t = before[2].cpu().numpy(), before[3].cpu().numpy()
    moved = 0
    for b, n in enumerate(P.lens):
        at = P.at[b]
        keep, moves = co.evict(w[at], t[at], budget[b], None if protect is None else protect[b])
        lens.append(keep)
        moved += len(moves)
        if moves:
            src, dst = (torch.as_tensor(at[[m[i] for m in moves]], device=DEV) for i in (0, 1))
            for x, y in zip(want, before):
                x[dst] = y[src]
    assert length_out.tolist() == lens
    if not in_place:
        assert P.length.tolist() == P.lens
    for x, y in zip(P.flat(), want):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))       # every bit of every slot, the others untouched
    return moved


EVICT_LENS = [0, 1, 2, 31, 1023, 1024, 1025, 3000]


@pytest.mark.parametrize("dt,kv,dh,page", [(BF, 2, 64, 16), (BF, 1, 8, 3), (FP, 1, 20, 7), (FP, 3, 128, 64), (BF, 1, 4, 1)])
@pytest.mark.parametrize("share", [0.0, 0.02, 0.5, 0.9, 1.0, 3.0])
def test_evict(dt, kv, dh, page, share):
    P = Pool(EVICT_LENS, page, kv, dh, dt, seed=15)
    budget = [int(share * n) for n in EVICT_LENS]
    moved = check_evict(P, budget, in_place=share != 0.5)
    assert moved > 0 or share in (0.0, 1.0, 3.0)


def test_evict_ties_and_values_that_are_no_numbers():
    P = Pool([500, 2000, 900], 16, 1, 64, BF, seed=16)
    g = np.random.default_rng(2)
    odd = np.array([0.0, -0.0, 1.0, np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45, 3.4e38, -1.0], np.float32)
    for b in range(3):
        P.flat()[2][torch.as_tensor(P.at[b], device=DEV)] = torch.as_tensor(odd[g.integers(0, len(odd), P.lens[b])], device=DEV)
    P.flat()[2][torch.as_tensor(P.at[2], device=DEV)] = 1.0                 # all alike: the first ones stay
    check_evict(P, [230, 1100, 400])


@pytest.mark.parametrize("budget", [[3, -5, 40, 700], [64, 64, 64, 64]])
def test_evict_with_protected_tokens(budget):
    P = Pool([10, 64, 65, 800], 8, 2, 64, FP, seed=17)
    check_evict(P, budget, protect=[5, 60, 0, 790])


def test_evict_of_long_requests():
    P = Pool([40000, 17000], 32, 1, 64, BF, seed=18, extra=0)
    check_evict(P, [9000, 16999])


def test_evict_of_more_requests_than_sms_and_a_loose_bound():
    lens = [(53 * b) % 97 for b in range(200)]
    check_evict(Pool(lens, 8, 1, 64, BF, seed=19), [b % 50 for b in range(200)], max_length=96 + 400)


def test_evict_with_a_page_that_is_not_there_moves_nothing_wrong():
    P = Pool([64, 64], 16, 1, 64, BF, seed=20)
    P.table[0, 1] = P.pages + 5
    before = P.copy()
    ctx = B_.Context(64, 2, 1, 64, 1, 1)
    ctx.d3tom_cache_evict(P.cache, i32([20, 64]), None, 2, 64, P.length)
    assert ctx.device_status() == B_.ERR_INVALID_ARG
    ctx.reset_device_status()
    other = np.setdiff1d(np.arange(len(before[2])), P.at[0])
    for x, y in zip(P.flat(), before):
        assert torch.equal(x[other].nan_to_num(99), y[other].nan_to_num(99))
    assert P.length.tolist() == [20, 64]


# ------------------------------------------------------------------ refusals
def test_refusals():
    P = Pool([20], 8, 2, 64, BF, seed=21)
    ctx = B_.Context(16, 2, 4, 64, 4, 32)
    q, out, k = randn((2, 4, 64), BF, 1), torch.zeros(2, 256, dtype=BF, device=DEV), randn((2, 2, 64), BF, 2)
    pos, c1 = i32(np.zeros((2, 3))), i32([0, 2])
    before = P.copy()

    def refused(status, fn, *a, **kw):
        with pytest.raises(B_.D3tomError) as e:
            fn(*a, **kw)
        assert e.value.status == status

    many = i32(np.zeros((20, 3)))
    rope = lambda spec, rows=2, kv=2, qq=q: ctx.d3tom_rope(spec, qq, k, pos if rows == 3 else many, rows, kv, torch.empty_like(qq),
                                                           torch.empty_like(k))
    for bad in (B_.RopeSpec([0, 0, 0]), B_.RopeSpec([16, 16, 1]), B_.RopeSpec([40]), B_.RopeSpec([-1, 5]), B_.RopeSpec([8], theta=0.5),
                B_.RopeSpec([8], theta=float("nan")), B_.RopeSpec([8], pairing=2), B_.RopeSpec([8], ladder=-1)):
        refused(B_.ERR_INVALID_ARG, rope, bad)
    refused(B_.ERR_WORKSPACE, rope, B_.RopeSpec([8]), 17)
    refused(B_.ERR_INVALID_ARG, rope, B_.RopeSpec([8]), -1)
    odd = torch.empty(2 * 4 * 64 + 1, dtype=BF, device=DEV)[1:].view(2, 4, 64)
    refused(B_.ERR_INVALID_ARG, rope, B_.RopeSpec([8]), 2, 2, odd)           # not 16-byte aligned

    def attn(cache=P.cache, q=q, rows=2, max_rows=2, max_length=20, scale=0.1, mode=0, out=out, B=1):
        ctx.d3tom_attn_cached(cache, q, c1, B, rows, max_rows, max_length, scale, mode, None, out)
    refused(B_.ERR_INVALID_ARG, attn, scale=0.0)
    refused(B_.ERR_INVALID_ARG, attn, scale=float("inf"))
    refused(B_.ERR_INVALID_ARG, attn, max_rows=3)
    refused(B_.ERR_INVALID_ARG, attn, max_length=-1)
    refused(B_.ERR_INVALID_ARG, attn, mode=3)
    refused(B_.ERR_INVALID_ARG, attn, B=0)
    refused(B_.ERR_WORKSPACE, ctx.d3tom_attn_cached, Pool([20, 1, 1], 8, 2, 64, BF).cache, q, i32([0, 2, 2, 2]), 3, 2, 2, 20, 0.1, 0, None, out)
    refused(B_.ERR_WORKSPACE, attn, rows=17)
    refused(B_.ERR_WORKSPACE, attn, mode=1, max_length=33)
    refused(B_.ERR_WORKSPACE, attn, mode=1, rows=5)
    refused(B_.ERR_INVALID_ARG, attn, q=odd)
    no_weight = B_.Cache(P.k, P.v, None, None, P.table, P.length)
    refused(B_.ERR_INVALID_ARG, attn, cache=no_weight, mode=1)
    three = Pool([20], 8, 3, 64, BF)
    refused(B_.ERR_INVALID_ARG, attn, cache=three.cache)                     # 4 heads do not share 3 key heads
    refused(B_.ERR_UNSUPPORTED, attn, cache=Pool([20], 12, 2, 64, BF).cache)  # bf16 pages of 12 slots
    small = B_.Context(16, 2, 4, 40, 4, 32)
    refused(B_.ERR_UNSUPPORTED, small.d3tom_attn_cached, Pool([20], 8, 2, 40, BF).cache, randn((2, 4, 40), BF, 1), c1, 1, 2, 2, 20, 0.1, 0,
            None, torch.zeros(2, 160, dtype=BF, device=DEV))
    refused(B_.ERR_INVALID_ARG, ctx.d3tom_cache_append, P.cache, B_.RopeSpec([8]), None, k, k, None, None, None, c1, 1, 2, None)
    refused(B_.ERR_INVALID_ARG, ctx.d3tom_cache_append, P.cache, None, q, k, k, None, None, None, c1, 1, 2, None)
    refused(B_.ERR_INVALID_ARG, ctx.d3tom_cache_append, no_weight, None, None, k, k, None, i32([1, 2]), None, c1, 1, 2, None)
    refused(B_.ERR_WORKSPACE, ctx.d3tom_cache_append, P.cache, None, None, k, k, None, None, None, c1, 1, 17, None)
    refused(B_.ERR_INVALID_ARG, ctx.d3tom_cache_evict, no_weight, i32([3]), None, 1, 20, P.length)
    refused(B_.ERR_INVALID_ARG, ctx.d3tom_cache_evict, B_.Cache(P.k, P.v, P.weight, None, P.table, P.length), i32([3]), i32([3]), 1, 20, P.length)
    refused(B_.ERR_WORKSPACE, ctx.d3tom_cache_evict, P.cache, i32([3]), None, 1, 16 * 4 * 64, P.length)
    with pytest.raises(TypeError):
        ctx.d3tom_attn_cached(P.cache, q.float(), c1, 1, 2, 2, 20, 0.1, 0, None, out)
    with pytest.raises(ValueError):
        B_.Cache(P.k, P.v, P.weight[:1], None, P.table, P.length)
    with pytest.raises(ValueError):
        ctx.d3tom_attn_cached(P.cache, q, i32([0, 1, 2]), 2, 2, 1, 20, 0.1, 0, None, out)      # the table has one request
    with pytest.raises(TypeError):
        ctx.d3tom_attn_cached(P.cache, q, c1[:1], 1, 2, 2, 20, 0.1, 0, None, out)
    with pytest.raises(TypeError):
        rope(B_.RopeSpec([1, 1, 1]), rows=3)                                 # positions of two rows
    with pytest.raises(TypeError):
        ctx.d3tom_cache_evict(P.cache, i32([3]).long(), None, 1, 20, P.length)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for x, y in zip(P.flat(), before):
        assert torch.equal(x.nan_to_num(99), y.nan_to_num(99))


# ------------------------------------------------------------------ together, as they are used
@pytest.mark.parametrize("dt,H,kv,dh,page", [(BF, 8, 2, 128, 16), (FP, 4, 4, 32, 6)])
def test_decoding_with_a_cache_that_shrinks(dt, H, kv, dh, page):
    """Prefix appended with positions, three denoising steps of a block: append, attend with this step's importance,
    drop the block, evict; against the same in fp64 on the host, which takes the cache's own stored numbers."""
    lens, block = [150, 61, 300], [5, 3, 0]
    spec, sec = B_.RopeSpec([dh // 8, dh // 8, dh // 4]), [dh // 8, dh // 8, dh // 4]
    C = PagedCache(3, H, kv, dh, dt, pages=sum(-(-n // page) for n in lens) + 3, page_size=page, max_rows=sum(lens), max_length=310,
                   max_scored_rows=8)
    total = sum(lens)
    rng = np.random.default_rng(4)
    pos = i32(rng.integers(0, 4000, (total, 3)))
    k, v = randn((total, kv, dh), dt, 1), randn((total, kv, dh), dt, 2)
    tok = np.concatenate([np.arange(n) for n in lens])
    first = torch.where(i32(tok) % 10 == 0, float("inf"), 0.0)               # prompt rows stay
    C.append(lens, k, v, i32(tok), spec=spec, positions=pos, first_weight=first)
    budget = [100, 61, 40]
    for step in range(3):
        n_new = sum(block)
        q, kb, vb = randn((n_new, H, dh), dt, 10 + step), randn((n_new, kv, dh), dt, 20 + step), randn((n_new, kv, dh), dt, 30 + step)
        pb = i32(rng.integers(4000, 5000, (n_new, 3)))
        q_rot, out = torch.empty_like(q), torch.empty(n_new, H * dh, dtype=dt, device=DEV)
        C.append(block, kb, vb, i32(np.arange(n_new) + 1000), q=q, q_out=q_rot, spec=spec, positions=pb)
        C.attend(block, q_rot, out, B_.WEIGHT_ADD)
        n_now = list(C.lengths_h)
        w = C.weight.view(-1).clone()
        for b in range(3):
            lo, hi = cu(block)[b], cu(block)[b + 1]
            at = co.places(C.table_h[b], n_now[b], page)
            idx = torch.as_tensor(at, device=DEV)
            ang = co.rope_angles(pb[lo:hi].cpu().numpy(), sec, 1e4, False)
            want_k = co.rope(f64(kb[lo:hi]), ang)
            assert (np.abs(f64(C.k.view(-1, kv, dh)[idx[n_now[b] - (hi - lo):]]) - want_k) <= HALF[dt] * np.abs(want_k) + 2e-5).all()
            o, p, mag, reach = co.attend(f64(q_rot[lo:hi]), f64(C.k.view(-1, kv, dh)[idx]), f64(C.v.view(-1, kv, dh)[idx]), dh ** -0.5)
            got = f64(out[lo:hi]).reshape(o.shape)
            assert (np.abs(got - o) <= HALF[dt] * np.abs(o) + ((2.0 ** -8 if dt == BF else 0) + 1e-4) * mag).all()
            prefix = C.token.view(-1)[idx]
            assert torch.isinf(w[idx][(prefix < 1000) & (prefix % 10 == 0)]).all()
        C.drop_last(block)
        wt, tk = C.weight.view(-1).cpu().numpy().copy(), C.token.view(-1).cpu().numpy().copy()
        expect = [co.evict(wt[co.places(C.table_h[b], C.lengths_h[b], page)], None, budget[b]) for b in range(3)]
        tokens = []
        for b in range(3):
            t = tk[co.places(C.table_h[b], C.lengths_h[b], page)].copy()
            for src, dst in expect[b][1]:
                t[dst] = t[src]
            tokens.append(t[: expect[b][0]])
        C.evict(budget)
        assert C.lengths_h == [e[0] for e in expect] == C.length.tolist() == [100, 61, 40]
        for b in range(3):
            at = co.places(C.table_h[b], C.lengths_h[b], page)
            got = C.token.view(-1).cpu().numpy()[at]
            assert np.array_equal(got, tokens[b])
            assert set(range(0, lens[b], 10)) <= set(got.tolist())           # the prompt is still there
    assert C.ctx.device_status() == 0
    with pytest.raises(RuntimeError):
        C.append([400, 0, 0], k, v, i32(tok))


@pytest.mark.parametrize("dt", [BF, FP])
def test_captured_step_follows_lengths_that_change(dt):
    """Append, attend and evict recorded once; replayed after the lengths and rows on the device have changed, beside a second
    context on another stream."""
    H, kv, dh, page = 4, 2, 64, 16
    lens = [90, 200]
    P = Pool(lens, page, kv, dh, dt, seed=22, extra=12)
    wide = np.full((2, 20), -1, np.int32)                                     # a table with room for 90 slots more
    wide[:, : P.table_h.shape[1]] = P.table_h
    used = set(P.table_h[P.table_h >= 0].tolist())
    spare = [p for p in range(P.pages) if p not in used]
    for b, n in enumerate(lens):
        for i in range(6):
            wide[b, -(-n // page) + i] = spare.pop()
    table, length = i32(wide), i32([n + 1 for n in lens])
    cache = B_.Cache(P.k, P.v, P.weight, P.token, table, length)
    ctxs = [B_.Context(64, 2, H, dh, 4, 320) for _ in range(2)]
    spec = B_.RopeSpec([16, 8])
    q, k, v = randn((2, H, dh), dt, 1), randn((2, kv, dh), dt, 2), randn((2, kv, dh), dt, 3)
    pos, tok, c = i32([[1, 2], [3, 4]]), i32([7000, 7001]), i32([0, 1, 2])
    q_rot, out, new = torch.empty_like(q), torch.empty(2, H * dh, dtype=dt, device=DEV), i32([0, 0])
    budget = i32([60, 150])

    def step(ctx):
        ctx.d3tom_cache_append(cache, spec, q, k, v, pos, tok, None, c, 2, 2, q_rot)
        ctx.d3tom_attn_cached(cache, q_rot, c, 2, 2, 1, 320, 0.125, B_.WEIGHT_ADD, None, out)

    side = torch.cuda.Stream()
    saved = P.copy()
    with torch.cuda.stream(side):
        step(ctxs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ctxs[0])
        ctxs[0].d3tom_cache_evict(cache, budget, None, 2, 320, new)
    for grow in (1, 17, 90):
        for x, y in zip(P.flat(), saved):
            x.copy_(y.nan_to_num(0.5) if x.is_floating_point() else y)
        now = [n + grow for n in lens]
        length.copy_(i32(now))
        q.copy_(randn((2, H, dh), dt, grow))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in P.flat()] + [out.clone(), q_rot.clone(), new.clone()]
        for x, y in zip(P.flat(), saved):
            x.copy_(y.nan_to_num(0.5) if x.is_floating_point() else y)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            step(ctxs[1])
            ctxs[1].d3tom_cache_evict(cache, budget, None, 2, 320, new)
        torch.cuda.synchronize()
        for x, y in zip(got, [*P.flat(), out, q_rot, new]):
            assert torch.equal(x, y)
        assert got[6].tolist() == [min(60, now[0]), min(150, now[1])]
    assert ctxs[0].device_status() == 0 and ctxs[1].device_status() == 0
