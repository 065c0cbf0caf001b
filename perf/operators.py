"""A key/value cache in pages and the operators around it, as cases that can be timed.

What a response block of a diffusion multimodal LLM needs once its [visual | prompt] prefix is cached:
  rope    rotary positions with up to three axes (time, height, width) for the rows of Q and K, and the way back
  append  K rotated and written with V, the token's number and its first weight into the pages of each request, Q rotated alike
  attn    attention of the new rows of each request over all of its cached slots; the attention mass that falls on a slot goes
          into that slot's weight
  evict   each request keeps its heaviest slots: kept slots from behind the new length move into the gaps before it
Values: rows N(0,1), a tenth of the cached keys moved by a shared direction per head that the queries lean to (a few slots draw most
of the weight, as visual tokens do), weights of a cache the squares of N(0,1).  ``own`` chooses between elementary torch operations
and the library's calls.
"""
import math

import numpy as np
import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # a response block of one request (the smallest call a denoising step makes)
        {"name": "rope_block", "op": "rope", "dtype": "bf16", "rows": 64, "heads": 32, "kv_heads": 32, "dh": 128,
         "sections": "16,24,24", "pairing": "halves", "ladder": "shared", "inverse": False, "far": False},
        # the whole [visual | prompt | response] sequence of one request
        {"name": "rope_sequence", "op": "rope", "dtype": "bf16", "rows": 4288, "heads": 32, "kv_heads": 32, "dh": 128,
         "sections": "16,24,24", "pairing": "halves", "ladder": "shared", "inverse": False, "far": False},
        # keys taken back to their unrotated form in 32 bits, neighbouring pairs, part of the head, far positions
        {"name": "rope_back_fp32", "op": "rope", "dtype": "fp32", "rows": 1153, "heads": 16, "kv_heads": 4, "dh": 64,
         "sections": "8,8,8", "pairing": "neighbours", "ladder": "per_axis", "inverse": True, "far": True},
        # one new token of each of 64 requests
        {"name": "append_tokens", "op": "append", "dtype": "bf16", "batch": 64, "rows": 1, "len": 2176, "len_min": 200, "heads": 32,
         "kv_heads": 8, "dh": 128, "page": 16, "sections": "16,24,24", "far": False},
        # the prefixes of a ragged batch, written for the first time
        {"name": "append_prefix", "op": "append", "dtype": "bf16", "batch": 8, "rows": 4352, "len": 4352, "len_min": 1056, "heads": 32,
         "kv_heads": 32, "dh": 128, "page": 64, "sections": "16,24,24", "far": False},
        # one token of one request on a merged sequence: latency
        {"name": "attn_one_short", "op": "attn", "dtype": "bf16", "batch": 1, "rows": 1, "len": 1216, "len_min": 1216, "heads": 32,
         "kv_heads": 32, "dh": 128, "page": 16, "weight": "none"},
        # serving: one token of each of 64 requests, shared key heads, weights accumulated
        {"name": "attn_batch", "op": "attn", "dtype": "bf16", "batch": 64, "rows": 1, "len": 8192, "len_min": 37, "heads": 32,
         "kv_heads": 8, "dh": 128, "page": 64, "weight": "add"},
        # a response block of each request over its cached prefix, importance of this step
        {"name": "attn_block", "op": "attn", "dtype": "bf16", "batch": 8, "rows": 32, "len": 4288, "len_min": 1088, "heads": 32,
         "kv_heads": 32, "dh": 128, "page": 48, "weight": "set"},
        # one token over a very long cache
        {"name": "attn_long", "op": "attn", "dtype": "bf16", "batch": 1, "rows": 1, "len": 131071, "len_min": 131071, "heads": 32,
         "kv_heads": 8, "dh": 128, "page": 16, "weight": "none"},
        # 32-bit cache, a few rows, odd sizes
        {"name": "attn_fp32", "op": "attn", "dtype": "fp32", "batch": 4, "rows": 3, "len": 2177, "len_min": 515, "heads": 16,
         "kv_heads": 4, "dh": 64, "page": 20, "weight": "add"},
        # serving: 32 requests a little over their budgets
        {"name": "evict_little", "op": "evict", "dtype": "bf16", "batch": 32, "len": 2112, "len_min": 2049, "budget": 2048, "kv_heads": 8,
         "dh": 128, "page": 16, "recent": 64},
        # prefixes cut to a quarter after the first step
        {"name": "evict_prefix", "op": "evict", "dtype": "bf16", "batch": 8, "len": 8192, "len_min": 1100, "budget": 1216, "kv_heads": 32,
         "dh": 128, "page": 64, "recent": 0},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attn", "attn", "evict"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    dh = rng.choice([64, 128])
    heads, kv = rng.choice([(32, 32), (32, 8), (16, 4), (28, 4), (12, 12), (8, 1)])
    pairs = rng.randint(1, dh // 2)
    a = rng.randint(0, pairs)
    b = rng.randint(0, pairs - a)
    sections = "%d,%d,%d" % (a, b, pairs - a - b)
    page = rng.choice([8, 16, 24, 32, 48, 64, 128])
    if op == "rope":
        return {"op": op, "dtype": dtype, "rows": _log(rng, 1, 4000 if dtype == "bf16" else 2000), "heads": heads, "kv_heads": kv,
                "dh": dh, "sections": sections, "pairing": rng.choice(["halves", "neighbours"]),
                "ladder": rng.choice(["shared", "per_axis"]), "inverse": rng.random() < 0.5, "far": rng.random() < 0.5}
    batch = _log(rng, 1, 48)
    most = max(16, int({"append": 16000, "attn": 60000, "evict": 40000}[op] / batch * (8.0 / kv if kv > 8 else 1.0)))
    if op == "append":
        n = _log(rng, 1, most)
        return {"op": op, "dtype": dtype, "batch": batch, "rows": min(n, 4000), "len": n + rng.randint(0, 500),
                "len_min": rng.randint(0, n), "heads": heads, "kv_heads": kv, "dh": dh, "page": page, "sections": sections,
                "far": rng.random() < 0.5}
    n = _log(rng, 16, most)
    if op == "evict":
        return {"op": op, "dtype": dtype, "batch": batch, "len": n, "len_min": rng.randint(0, n), "budget": rng.randint(1, n),
                "kv_heads": kv, "dh": dh, "page": page, "recent": rng.choice([0, 0, 1, 32])}
    return {"op": op, "dtype": dtype, "batch": batch, "rows": _log(rng, 1, 40 if dtype == "bf16" else 8), "len": n,
            "len_min": rng.randint(0, n), "heads": heads, "kv_heads": kv, "dh": dh, "page": page,
            "weight": rng.choice(["none", "add", "set"])}


def _lens(case):
    """Lengths of the requests, spread over [len_min, len] out of order; the same for every seed."""
    B, lo, hi = case["batch"], case["len_min"], case["len"]
    if B == 1:
        return [hi]
    return [lo + ((b * 5 + 2) % B) * (hi - lo) // (B - 1) if B % 5 else lo + ((b * 3 + 1) % B) * (hi - lo) // (B - 1) for b in range(B)]


def _new_rows(case):
    """New rows of the requests: a block is as long as its request allows."""
    return [min(case["rows"], n) for n in _lens(case)]


def _sections(case):
    return [int(x) for x in case["sections"].split(",")]


def _positions(total, far, gen):
    """Time, height and width of the rows: a grid of 24 columns; far ones start at a million."""
    i = torch.arange(total, device="cuda")
    start = torch.randint(0, 500, (3,), generator=gen, device="cuda") + (1000003 if far else 0)
    return torch.stack([start[0] + i // 576, start[1] + i // 24 % 24, start[2] + i % 24], dim=1).to(torch.int32).contiguous()


def _table(lens, page, extra, gen):
    """Every request's pages, drawn from the pool out of order; entries behind a request's last page stay -1."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + extra
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    width = max(1, max(need))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(need)]), device="cuda")
    j = torch.arange(width, device="cuda")[None, :]
    n = torch.tensor(need, device="cuda")[:, None]
    at = (cu[:-1, None] + j).clamp(max=pages - 1)
    return torch.where(j < n, order[at], torch.full_like(order[at], -1)).contiguous(), pages


def _cu(a):
    return torch.tensor(np.concatenate([[0], np.cumsum(a)]).astype(np.int32), device="cuda")


def _randn(shape, dt, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dt)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": case, "dt": _DT[case["dtype"]]}
    op, dt, dh, kv = case["op"], st["dt"], case["dh"], case["kv_heads"]
    if op == "rope":
        n, H = case["rows"], case["heads"]
        st["q"], st["k"] = _randn((n, H, dh), dt, gen), _randn((n, kv, dh), dt, gen)
        st["pos"] = _positions(n, case["far"], gen)
        st["q_out"], st["k_out"] = torch.empty_like(st["q"]), torch.empty_like(st["k"])
        if own:
            _own_state(st, n, 1, H, dh, 1, 1)
        return st
    lens, page = _lens(case), case["page"]
    B, L = case["batch"], max(lens)
    st["lens"], st["L"] = lens, L
    st["table"], pages = _table(lens, page, 3, gen)
    st["pages"] = pages
    # one page more than the pool has: where the plain forms put what goes nowhere
    st["k_all"] = torch.empty((pages + 1, page, kv, dh), device="cuda", dtype=dt)
    st["v_all"] = torch.empty_like(st["k_all"])
    for t in (st["k_all"], st["v_all"]):
        for part in t.split(max(1, (1 << 27) // (page * kv * dh))):
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    st["w_all"] = torch.randn((pages + 1, page), generator=gen, device="cuda").square()
    st["token_all"] = torch.randint(0, 1 << 20, (pages + 1, page), generator=gen, device="cuda", dtype=torch.int32)
    st["length"] = torch.tensor(lens, device="cuda", dtype=torch.int32)
    if op in ("append", "attn"):
        H, rows = case["heads"], _new_rows(case)
        T = max(1, sum(rows))
        st["rows"], st["total"] = rows, sum(rows)
        st["cu_rows"] = _cu(rows)
        st["q"] = _randn((T, H, dh), dt, gen)
    if op == "append":
        st["k"], st["v"] = _randn((T, kv, dh), dt, gen), _randn((T, kv, dh), dt, gen)
        st["pos"] = _positions(T, case["far"], gen)
        first = torch.repeat_interleave(torch.tensor([n - r for n, r in zip(lens, rows)], device="cuda"), torch.tensor(rows, device="cuda"))
        begin = torch.repeat_interleave(st["cu_rows"][:-1].long(), torch.tensor(rows, device="cuda"))
        tok = torch.zeros(T, device="cuda", dtype=torch.int32)
        tok[: sum(rows)] = (first + torch.arange(sum(rows), device="cuda") - begin).to(torch.int32)
        st["tokens"] = tok
        # prompt rows are never evicted: their weight is infinite from the start
        st["first_weight"] = torch.where(torch.arange(T, device="cuda") % 7 == 0, math.inf, 0.0).to(torch.float32)
        st["q_out"] = torch.empty_like(st["q"])
    if op == "attn":
        lean = torch.randn((kv, dh), generator=gen, device="cuda")
        lean = 4.0 * lean / lean.norm(dim=1, keepdim=True)
        hit = torch.rand((pages + 1, page, 1, 1), generator=gen, device="cuda") < 0.1
        for part, h in zip(st["k_all"].split(4096), hit.split(4096)):
            part.copy_(part.float() + h * lean)
        st["q"].copy_((st["q"].float().view(T, kv, H // kv, dh) + lean[None, :, None]).view(T, H, dh))
        st["out"] = torch.zeros((T, H * dh), device="cuda", dtype=dt)
        # rows that decide (the tokens decoded last) count in full, the others less
        st["row_weight"] = torch.rand(T, generator=gen, device="cuda") if case["weight"] == "set" else None
    if op == "evict":
        st["w_start"] = st["w_all"].clone()
        st["budget"] = torch.tensor([max(0, case["budget"] - b % 3) for b in range(B)], device="cuda", dtype=torch.int32)
        st["length_out"] = torch.zeros_like(st["length"])
        if case["recent"]:
            # tokens numbered by slot: the last ones of a request are protected
            slot = torch.arange(st["table"].shape[1] * page, device="cuda")
            flat, ok = _slots(st, slot.numel())
            st["token_all"].view(-1)[flat[ok]] = slot.to(torch.int32).expand(B, -1)[ok]
            st["protect_from"] = (st["length"] - case["recent"]).to(torch.int32)
        else:
            st["protect_from"] = None
    if own:
        H = case.get("heads", kv)
        rows = max(1, st.get("total", 1))
        scored = rows if case.get("weight", "none") != "none" else 1
        tokens = max(rows, -(-B * (L + 2) // (H * dh)))
        _own_state(st, tokens, B, H, dh, scored, L if scored > 1 or case.get("weight", "none") != "none" else 1)
    return st


def _own_state(st, tokens, B, H, dh, scored, L):
    """The context, the cache and the rotary description that a user's program keeps."""
    from paper_2511_12280_b200 import binding as B_
    case = st["case"]
    st["ctx"] = B_.Context(tokens, B, H, dh, max(1, scored), max(1, L))
    if "sections" in case:
        sec = _sections(case)
        st["spec"] = B_.RopeSpec(sec, theta=10000.0,
                                 pairing=B_.PAIR_NEIGHBOURS if case.get("pairing") == "neighbours" else B_.PAIR_HALVES,
                                 ladder=B_.LADDER_PER_AXIS if case.get("ladder") == "per_axis" else B_.LADDER_SHARED)
    if case["op"] != "rope":
        n = st["pages"]
        st["cache"] = B_.Cache(st["k_all"][:n], st["v_all"][:n], st["w_all"][:n], st["token_all"][:n], st["table"], st["length"])


# ------------------------------------------------------------------ one pass
def run(st):
    return {"rope": _run_rope, "append": _run_append, "attn": _run_attn, "evict": _run_evict}[st["case"]["op"]](st)


def _slots(st, L):
    """[B, L] flat slot numbers in the pool (the spare page's where there is none) and which of them a request has."""
    page, table = st["case"]["page"], st["table"]
    slot = torch.arange(L, device="cuda")
    pg = table[:, (slot // page).clamp(max=table.shape[1] - 1)].long()
    ok = slot[None, :] < st["length"][:, None]
    spare = st["pages"] * page
    return torch.where(ok, pg * page + slot % page, torch.full_like(pg, spare)), ok


def _angles(case, pos):
    """Angle of every rotated pair, in 64 bits: positions go far beyond what 32 bits turn exactly."""
    sec = _sections(case)
    n = sum(sec)
    axis = torch.cat([torch.full((s,), a, device="cuda") for a, s in enumerate(sec)]).long()
    if case.get("ladder") == "per_axis":
        power = torch.cat([torch.arange(s, device="cuda", dtype=torch.float64) / max(1, s) for s in sec])
    else:
        power = torch.arange(n, device="cuda", dtype=torch.float64) / n
    return pos.double()[:, axis] * torch.pow(torch.tensor(10000.0, device="cuda", dtype=torch.float64), -power)


def _rotate(case, x, angle, inverse):
    n = angle.shape[1]
    c, s = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    s = -s if inverse else s
    y = x.float()
    if case.get("pairing") == "neighbours":
        a, b = y[..., 0 : 2 * n : 2], y[..., 1 : 2 * n : 2]
        rot = torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n : 2 * n]
        rot = torch.cat([a * c - b * s, a * s + b * c], dim=-1)
    return torch.cat([rot, y[..., 2 * n :]], dim=-1).to(x.dtype)


def _run_rope(st):
    case = st["case"]
    if own:
        st["ctx"].d3tom_rope(st["spec"], st["q"], st["k"], st["pos"], case["rows"], case["kv_heads"], st["q_out"], st["k_out"],
                             inverse=case["inverse"])
        return st["q_out"], st["k_out"]
    angle = _angles(case, st["pos"])
    return _rotate(case, st["q"], angle, case["inverse"]), _rotate(case, st["k"], angle, case["inverse"])


def _run_append(st):
    case, n = st["case"], st["pages"]
    outs = st["k_all"][:n], st["v_all"][:n], st["w_all"][:n], st["token_all"][:n]
    if own:
        st["ctx"].d3tom_cache_append(st["cache"], st["spec"], st["q"], st["k"], st["v"], st["pos"], st["tokens"], st["first_weight"],
                                     st["cu_rows"], case["batch"], st["total"], st["q_out"])
        return (st["q_out"][: st["total"]],) + outs
    angle = _angles(case, st["pos"])
    row = torch.arange(st["q"].shape[0], device="cuda")
    b = (torch.searchsorted(st["cu_rows"], row.to(torch.int32), right=True) - 1).clamp(max=case["batch"] - 1)
    slot = st["length"][b] - st["cu_rows"][b + 1] + row
    page = st["table"][b, (slot // case["page"]).clamp(0, st["table"].shape[1] - 1)].long()
    at = torch.where(row < st["total"], page * case["page"] + slot % case["page"], n * case["page"])
    st["k_all"].view(-1, case["kv_heads"], case["dh"])[at] = _rotate(case, st["k"], angle, False)
    st["v_all"].view(-1, case["kv_heads"], case["dh"])[at] = st["v"]
    st["w_all"].view(-1)[at] = st["first_weight"]
    st["token_all"].view(-1)[at] = st["tokens"]
    return (_rotate(case, st["q"], angle, False)[: st["total"]],) + outs


def _run_attn(st):
    case, n = st["case"], st["pages"]
    scale = 1.0 / math.sqrt(case["dh"])
    if own:
        from paper_2511_12280_b200 import binding as B_
        mode = {"none": B_.WEIGHT_NONE, "add": B_.WEIGHT_ADD, "set": B_.WEIGHT_SET}[case["weight"]]
        st["ctx"].d3tom_attn_cached(st["cache"], st["q"], st["cu_rows"], case["batch"], st["total"], max(st["rows"]), st["L"], scale,
                                    mode, st["row_weight"], st["out"])
        return st["out"][: st["total"]], st["w_all"][:n]
    B, H, kv, dh, L, N = case["batch"], case["heads"], case["kv_heads"], case["dh"], st["L"], case["rows"]
    at, ok = _slots(st, L)
    k = st["k_all"].view(-1, kv, dh)[at].float()
    q_row = st["cu_rows"][:-1, None].long() + torch.arange(N, device="cuda")
    has = torch.arange(N, device="cuda")[None, :] < (st["cu_rows"][1:] - st["cu_rows"][:-1])[:, None]
    q_row = torch.where(has, q_row, torch.zeros_like(q_row))
    q = st["q"][q_row].float().view(B, N, kv, H // kv, dh).permute(0, 2, 3, 1, 4).reshape(B, kv, H // kv * N, dh)
    s = torch.matmul(q, k.permute(0, 2, 3, 1)) * scale
    del k
    s = s.masked_fill(~ok[:, None, None, :], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    del s
    l = p.sum(dim=-1, keepdim=True)
    p /= torch.where(l == 0, 1.0, l)
    v = st["v_all"].view(-1, kv, dh)[at].masked_fill(~ok[:, :, None, None], 0).float()
    o = torch.matmul(p, v.permute(0, 2, 1, 3)).view(B, kv, H // kv, N, dh).permute(0, 3, 1, 2, 4).reshape(B * N, H * dh)
    del v
    # rows of the padded block back to the packed ones; rows that no request has go to a row of their own
    T = st["q"].shape[0]
    out = torch.zeros((T + 1, H * dh), device="cuda", dtype=st["dt"])
    out[torch.where(has, q_row, T).view(-1)] = o.to(st["dt"])
    if case["weight"] != "none":
        f = has.float() if st["row_weight"] is None else has * st["row_weight"][q_row]
        mass = (p.view(B, kv * (H // kv), N, L) * f[:, None, :, None]).sum(dim=(1, 2))
        w = st["w_all"].view(-1)
        w[at.view(-1)] = (mass + w[at] if case["weight"] == "add" else mass).view(-1)
    return out[: st["total"]], st["w_all"][:n]


def _run_evict(st):
    case, n = st["case"], st["pages"]
    st["w_all"].copy_(st["w_start"])     # the weights of this step (a pass leaves the moved ones behind)
    outs = st["k_all"][:n], st["v_all"][:n], st["w_all"][:n], st["token_all"][:n], st["length_out"]
    if own:
        st["ctx"].d3tom_cache_evict(st["cache"], st["budget"], st["protect_from"], case["batch"], st["L"], st["length_out"])
        return outs
    B, kv, dh, L = case["batch"], case["kv_heads"], case["dh"], st["L"]
    at, ok = _slots(st, L)
    w, tok = st["w_all"].view(-1), st["token_all"].view(-1)
    key = w[at]
    if st["protect_from"] is not None:
        key = torch.where(tok[at] >= st["protect_from"][:, None], math.nan, key)     # ranks before every number
    key = torch.where(ok, key, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, torch.arange(L, device="cuda").expand(B, -1))
    new = torch.minimum(st["budget"].clamp(min=0), st["length"])[:, None]
    slot = torch.arange(L, device="cuda")[None, :]
    kept = (rank < new) & ok
    gap, mover = (slot < new) & ~kept, (slot >= new) & kept
    spare = n * case["page"]
    src = torch.full((B, L + 1), spare, device="cuda", dtype=torch.int64)
    src.scatter_(1, torch.where(mover, mover.cumsum(1) - 1, L), torch.where(mover, at, spare))
    frm = torch.where(gap, src.gather(1, (gap.cumsum(1) - 1).clamp(min=0)), spare).view(-1)
    to = torch.where(gap, at, spare).view(-1)
    for t in (st["k_all"].view(-1, kv, dh), st["v_all"].view(-1, kv, dh), w, tok):
        t[to] = t[frm]
    st["length_out"].copy_(new[:, 0])
    return outs


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    kv, dh = case["kv_heads"], case["dh"]
    if case["op"] == "rope":
        n = case["rows"] * (case["heads"] + kv) * dh
        return {"bytes": 2 * n * size + case["rows"] * 12, "flops": 3 * n}
    lens = _lens(case)
    if case["op"] == "evict":
        # weights and tokens read; at most the slots over the budget move, in expectation this share of the kept ones
        total = bytes_moved = 0
        for b, n in enumerate(lens):
            k = min(n, max(0, case["budget"] - b % 3))
            total += n
            bytes_moved += k * (n - k) / max(1, n) * (2 * kv * dh * size + 8) * 2
        return {"bytes": total * (8 if case["recent"] else 4) + bytes_moved, "flops": total}
    rows = _new_rows(case)
    if case["op"] == "append":
        n = sum(rows)
        return {"bytes": 2 * n * (case["heads"] + 2 * kv) * dh * size + n * 28, "flops": 3 * n * (case["heads"] + kv) * dh}
    H = case["heads"]
    b = sum(2 * n * kv * dh * size for n, r in zip(lens, rows) if r) + 2 * sum(rows) * H * dh * size
    b += 0 if case["weight"] == "none" else sum(lens) * (8 if case["weight"] == "add" else 4)
    return {"bytes": b, "flops": sum(4 * n * r for n, r in zip(lens, rows)) * H * dh}


# ------------------------------------------------------------------ the definitions in 64 bits, request by request
def _turned(case, x, pos, inverse):
    """Every pair (a, b) as the complex number a + ib, times exp(+-i angle)."""
    sec, n = _sections(case), sum(_sections(case))
    f = []
    for i in range(n):
        ax = 0 if i < sec[0] else 1 if i < sec[0] + sec[1] else 2
        e = (i - sum(sec[:ax])) / sec[ax] if case.get("ladder") == "per_axis" else i / n
        f.append((ax, 10000.0 ** -e))
    phase = pos.cpu().numpy().astype(np.float64)[:, [a for a, _ in f]] * np.array([g for _, g in f])
    turn = torch.from_numpy(np.exp((-1j if inverse else 1j) * phase)).cuda()[:, None, :]
    y = x.double().clone()
    if case.get("pairing") == "neighbours":
        z = torch.view_as_complex(y[..., : 2 * n].unflatten(-1, (n, 2)).contiguous()) * turn
        y[..., : 2 * n] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(y[..., :n], y[..., n : 2 * n]) * turn
        y[..., :n], y[..., n : 2 * n] = z.real, z.imag
    return y


def _where(st, b, n):
    page = st["case"]["page"]
    t = st["table"][b].cpu().numpy().astype(np.int64)
    j = np.arange(n)
    return torch.from_numpy(t[j // page] * page + j % page).cuda()


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return _turned(case, st["q"], st["pos"], case["inverse"]), _turned(case, st["k"], st["pos"], case["inverse"])
    n, kv, dh = st["pages"], case["kv_heads"], case["dh"]
    k, v = st["k_all"][:n].reshape(-1, kv, dh), st["v_all"][:n].reshape(-1, kv, dh)
    w, tok = st["w_all"][:n].reshape(-1).double(), st["token_all"][:n].reshape(-1).clone()
    if case["op"] == "append":
        k, v = k.double(), v.double()
        cu = st["cu_rows"].tolist()
        for b, size in enumerate(st["lens"]):
            lo, hi = cu[b], cu[b + 1]
            at = _where(st, b, size)[size - (hi - lo) :]
            k[at] = _turned(case, st["k"][lo:hi], st["pos"][lo:hi], False)
            v[at] = st["v"][lo:hi].double()
            w[at] = st["first_weight"][lo:hi].double()
            tok[at] = st["tokens"][lo:hi]
        q = _turned(case, st["q"][: st["total"]], st["pos"][: st["total"]], False)
        return q, k.view_as(st["k_all"][:n]), v.view_as(st["k_all"][:n]), w.view_as(st["w_all"][:n]), tok.view_as(st["token_all"][:n])
    if case["op"] == "attn":
        H, cu = case["heads"], st["cu_rows"].tolist()
        out = torch.zeros((st["total"], H * dh), device="cuda", dtype=torch.float64)
        for b, size in enumerate(st["lens"]):
            lo, hi = cu[b], cu[b + 1]
            at = _where(st, b, size)
            mass = torch.zeros(size, device="cuda", dtype=torch.float64)
            for g in range(kv if size and hi > lo else 0):
                qs = st["q"][lo:hi, g * (H // kv) : (g + 1) * (H // kv)].double()
                a = torch.softmax(torch.einsum("rhd,jd->rhj", qs, k[at, g].double()) / math.sqrt(dh), dim=-1)
                o = torch.einsum("rhj,jd->rhd", a, v[at, g].double())
                out[lo:hi].view(hi - lo, H, dh)[:, g * (H // kv) : (g + 1) * (H // kv)] = o
                f = torch.ones(hi - lo, device="cuda") if st["row_weight"] is None else st["row_weight"][lo:hi]
                mass += torch.einsum("rhj,r->j", a, f.double())
            if case["weight"] != "none":
                w[at] = mass + (w[at] if case["weight"] == "add" else 0.0)
        return out, w.view_as(st["w_all"][:n])
    length = []
    for b, size in enumerate(st["lens"]):
        at = _where(st, b, size)
        keep = min(size, max(0, case["budget"] - b % 3))
        ws, ts = w[at].cpu().numpy(), tok[at].cpu().numpy()
        safe = ts >= int(st["protect_from"][b]) if st["protect_from"] is not None else np.zeros(size, bool)
        best = np.lexsort((np.arange(size), -ws, ~safe))[:keep]
        gaps = np.setdiff1d(np.arange(keep), best)
        movers = np.sort(best[best >= keep])
        to, frm = at[torch.from_numpy(gaps).cuda()], at[torch.from_numpy(movers).cuda()]
        for t in (k, v, w, tok):
            t[to] = t[frm]
        length.append(keep)
    shape = st["k_all"][:n].shape
    return k.view(shape), v.view(shape), w.view_as(st["w_all"][:n]), tok.view_as(st["token_all"][:n]), torch.tensor(length)
