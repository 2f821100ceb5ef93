"""Folds of many sequences at once, on a cache in pages, as measurable cases.

Three operators, each reached through the package's public entry points:

* "assign": where the new tokens of a batch of requests go, found on the GPU from the requests' lengths (`KvFoldPagedCache.assign`).  Request s
  holds lens[s] tokens, on ceil(lens[s] / page) pages named by its row of the table, and gets new[s] more.  Pages that it lacks come from the end of the free
  list, in the order of the requests: with `first` the pages that requests before it lack, its j-th is free[n_free - 1 - first - j].  Results: the table, the lengths
  after, the running sum of the new tokens, for every token its place page * page_tokens + row and its position (-1 behind the last token), the
  free pages left, and a status: 1 more pages needed than free, 2 a row of the table too short, 4 more tokens than places asked
  for, 8 a count below zero, added up.  Where it is not 0 nothing is assigned: no request has new tokens.
* "decode": a fold step of one token, or a few, of every sequence (`KvFoldPagedCache.step`): the new K and V rows are written to their places, then query row i
  of a sequence that had prev tokens attends to rows j <= prev + i, found by its row of the table.
* "prompt": the same call for whole prompts, prev = 0, and for chunks of prompts: sequences of different lengths, their new tokens packed one
  sequence behind the other.

Keys of a case: op, dtype ("bf16" or "f32"), hq / hkv / d (query heads, KV heads, head dim), page (tokens of a page), seqs, and the range
of prev and of new tokens of a sequence, prev_lo / prev_hi / new_lo / new_hi, spread over their logarithm by `spread` (_sizes); pad (rows
behind the last sequence), fused (q, k and v are parts of one tensor, as a fused projection leaves them), short (assign: pages that the free list lacks).
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _case(name, op, dtype="bf16", hq=32, hkv=8, d=128, page=64, seqs=1, prev=(0, 0), new=(1, 1), spread=1, pad=0, fused=False, short=0):
    case = {"name": name, "op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "page": page, "seqs": seqs, "prev_lo": prev[0], "prev_hi": prev[1],
            "new_lo": new[0], "new_hi": new[1], "spread": spread, "pad": pad, "fused": fused, "short": short}
    if name is None:
        del case["name"]
    return case


def listed():
    return [
        # A tick of a serving loop: 64 requests get a token each; the smallest call.
        _case("assign_tick_64", "assign", seqs=64, prev=(16, 8192), new=(1, 1), pad=0),
        # Prompts admitted in one go, small pages, the places of the whole batch.
        _case("assign_admit_300", "assign", page=16, seqs=300, prev=(0, 2048), new=(1, 4096), pad=37),
        # Decoding for one user, a short conversation: latency counts.
        _case("decode_1_of_300", "decode", seqs=1, prev=(300, 300)),
        # A serving batch of conversations of all lengths, rows from a fused projection.
        _case("decode_64_ragged", "decode", page=64, seqs=64, prev=(16, 16384), fused=True),
        # A full batch on small pages; memory.
        _case("decode_256_of_4k", "decode", page=16, seqs=256, prev=(3000, 5000), pad=8),
        # A few long documents, after their chains.
        _case("decode_4_of_128k", "decode", page=256, seqs=4, prev=(126000, 131000)),
        # Drafted tokens checked four at a time (16 rows a KV head).
        _case("decode_draft_32_of_8k", "decode", page=32, seqs=32, prev=(2000, 16000), new=(4, 4)),
        # fp32, the heads of the smallest workload.
        _case("decode_tiny_f32", "decode", dtype="f32", hq=4, hkv=1, d=64, page=16, seqs=8, prev=(1, 700)),
        # Prompts of a batch, packed: one token to some thousands.
        _case("prompt_16_packed", "prompt", seqs=16, new=(1, 6000), spread=3, pad=11),
        # One long prompt in one call; the largest.
        _case("prompt_16k", "prompt", page=128, seqs=1, new=(16384, 16384), fused=True),
        # A step of eight chains of 256-token chunks, at different depths, the sweep's heads.
        _case("prompt_8_chunks_c256", "prompt", hq=28, hkv=4, page=64, seqs=8, prev=(4096, 65536), new=(256, 256)),
        # fp32 prompts of no round length, 64-wide heads.
        _case("prompt_6_f32_d64", "prompt", dtype="f32", hq=8, hkv=2, d=64, page=32, seqs=6, new=(33, 900)),
    ]


# Head shapes of the repository's configurations and tests: (query heads, KV heads, head dim).
_SHAPES = ((32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 8, 64), (4, 1, 64), (8, 2, 128), (16, 2, 64))


def _log_uniform(rng, lo, hi):
    if hi <= lo:
        return lo
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(max(lo, 0.7)), math.log(hi + 1)))))))


def _sizes(case):
    """(tokens held, new tokens) of every sequence."""
    rng = random.Random(case["spread"] * 1009 + case["seqs"])
    return ([_log_uniform(rng, case["prev_lo"], case["prev_hi"]) if case["prev_hi"] else 0 for _ in range(case["seqs"])],
            [_log_uniform(rng, case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])])


def _cost(case):
    """Rough seconds of a pass, for keeping drawn cases no larger than the largest listed one."""
    w = work(case)
    return max(w["flops"] / (1e15 if case["dtype"] == "bf16" else 1e14), w["bytes"] / 5e12)


def draw(rng):
    limit = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("assign", "decode", "decode", "decode", "prompt", "prompt", "prompt"))
        hq, hkv, d = rng.choice(_SHAPES)
        case = dict(hq=hq, hkv=hkv, d=d, page=rng.choice((16, 32, 64, 128, 256)), spread=rng.randint(1, 10 ** 6), pad=rng.choice((0, 0, rng.randint(1, 40))),
                    dtype=rng.choice(("bf16", "bf16", "bf16", "bf16", "f32")), fused=rng.random() < 0.3)
        hi = _log_uniform(rng, 16, 131072)
        lo = _log_uniform(rng, 1, hi)
        if op == "assign":
            case.update(seqs=_log_uniform(rng, 1, 2000), prev=(0, hi), new=(rng.choice((0, 1)), _log_uniform(rng, 1, 4096)), short=rng.choice((0, 0, 0, 1)))
        elif op == "decode":
            few = max(1, 16 // (hq // hkv))  # (tokens of a sequence that a KV head's 16 rows hold)
            new = rng.choice((1, 1, rng.randint(1, few)))
            case.update(seqs=_log_uniform(rng, 1, 256), prev=(lo, hi), new=(rng.choice((new, rng.randint(0, new))), new))
        else:
            top = _log_uniform(rng, 17, 16384)
            case.update(seqs=_log_uniform(rng, 1, 64), prev=rng.choice(((0, 0), (0, 0), (lo, hi))), new=(rng.choice((0, 1, top)), top))
        case = _case(None, op, **case)
        prev, new = _sizes(case)
        if op == "assign":
            if 0 < sum(new) <= 1 << 20:
                return case
        elif sum(new) and sum(prev) + sum(new) <= 1 << 20 and max(p + n for p, n in zip(prev, new)) <= 132000 and _cost(case) <= limit:
            return case


def work(case):
    """Assign: lengths, new tokens, the pages taken, and every result written once.  Steps: every cached row that is seen, q, the new rows read and written,
    output and log-sum-exp; two products over the visible (row, key) pairs."""
    prev, new = _sizes(case)
    total = sum(new)
    if case["op"] == "assign":
        page = case["page"]
        taken = sum(-(-(p + n) // page) - -(-p // page) for p, n in zip(prev, new))
        return {"bytes": 16.0 * case["seqs"] + 8.0 * taken + 12.0 * (total + case["pad"]), "flops": 0.0}
    es = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d = (case[k] for k in ("hq", "hkv", "d"))
    seen = sum(p for p, n in zip(prev, new) if n)
    pairs = sum(n * (p + (n + 1) / 2.0) for p, n in zip(prev, new))
    return {"bytes": es * (2.0 * hkv * d * seen + 4.0 * hkv * d * total + 2.0 * hq * d * total) + 4.0 * hq * total, "flops": 4.0 * hq * d * pairs}


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 20260512)
    return gen


def _pages(case, gen):
    """What a serving loop holds: the free list, pages in no order, and the requests' rows of the table."""
    prev, new = _sizes(case)
    page = case["page"]
    held = [-(-p // page) for p in prev]
    after = [-(-(p + n) // page) for p, n in zip(prev, new)]
    n_pages = sum(after) + 5
    width = max(max(after), 1) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    # (entries of a row behind its pages name none)
    columns = torch.arange(width, device="cuda")
    counts = torch.tensor(held, device="cuda")
    first = counts.cumsum(0) - counts
    tables = torch.where(columns < counts[:, None], order[(first[:, None] + columns).clamp_max(n_pages - 1)], -1).to(torch.int32)
    free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    left = order[sum(held):]
    free[:left.numel()] = left
    return {"tables": tables, "free": free, "n_free": max(0, left.numel() - (5 + case["short"] if case["short"] else 0)), "n_pages": n_pages,
            "lens": torch.tensor(prev, dtype=torch.int32, device="cuda"), "new": torch.tensor(new, dtype=torch.int32, device="cuda")}


def _inputs(case, seed):
    """Tables, and for a step the pages with the rows held, q and the new rows, from the seed alone.  Keys have channels of different sizes, as a model's have."""
    gen = _generator(seed)
    x = _pages(case, gen)
    x["n_free"] = torch.tensor([x["n_free"]], dtype=torch.int32, device="cuda")
    if case["op"] == "assign":
        return x
    hq, hkv, d, page = (case[k] for k in ("hq", "hkv", "d", "page"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    x["tables"], x["lens"], x["cu"], x["slots"], _, _, _ = _plain_assign(case, x)
    rows = x["slots"].numel()
    gain = torch.exp(0.4 * torch.randn((hkv, 1, d), generator=gen, device="cuda"))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dt)

    x["k_pages"], x["v_pages"] = (normal(x["n_pages"], hkv, page, d) for _ in range(2))
    x["k_pages"].mul_(gain.to(dt))
    if case["fused"]:
        together = normal(rows, (hq + 2 * hkv) * d)
        x["q"], x["k"], x["v"] = (t.unflatten(1, (-1, d)) for t in together.split((hq * d, hkv * d, hkv * d), 1))
    else:
        x["q"], x["k"], x["v"] = (normal(rows, heads, d) for heads in (hq, hkv, hkv))
    x["k"].mul_(gain.transpose(0, 1).to(dt))
    return x


def prepare(case, seed):
    """The inputs, and what a serving program keeps: the pages, the batch with its tables and workspace, room for the results."""
    x = _inputs(case, seed)
    prev, new = _sizes(case)
    state = {"case": case, "x": x, "prev": prev, "new": new}
    most = {"max_new": max(max(new), 1), "max_len": max(p + n for p, n in zip(prev, new))}
    rows = sum(new) + case["pad"]
    if case["op"] == "assign":
        if own:
            from paper_2605_12471_amd import KvFoldBatch, KvFoldPagedCache
            state["cache"] = KvFoldPagedCache(1, 1, 1, 64, case["page"], x["n_pages"])
            state["batch"] = KvFoldBatch(state["cache"], x["tables"], rows, **most)
        return state
    state["out"] = torch.zeros((rows, case["hq"], case["d"]), dtype=x["q"].dtype, device="cuda")
    state["lse"] = torch.zeros((case["hq"], rows), device="cuda")
    if own:
        from paper_2605_12471_amd import KvFoldBatch, KvFoldPagedCache
        cache = KvFoldPagedCache(1, case["hq"], case["hkv"], case["d"], case["page"], x["n_pages"], case["dtype"])
        state["pages"] = cache.view(0)
        for name, pages in zip(("k", "v"), state["pages"]):
            pages.copy_(x.pop(name + "_pages"))
        one_each = max(new) == min(new) == 1 and not case["pad"]
        state["cache"] = cache
        state["batch"] = KvFoldBatch(cache, x["tables"], rows, lens=x["lens"], cu_new=x["cu"], slots=x["slots"], one_each=one_each, **most)
    return state


def run(state):
    case, x = state["case"], state["x"]
    if own:
        batch = state["batch"]
        if case["op"] == "assign":
            state["cache"].assign(batch, x["lens"], x["new"], x["free"], x["n_free"])
            return [batch.tables, batch.lens, batch.cu_new, batch.slots, batch.positions, batch.n_free, batch.status]
        state["cache"].step(0, batch, x["q"], x["k"], x["v"], state["out"], lse=state["lse"])
        return {"out": state["out"], "lse": state["lse"], "pages": state["pages"]}
    if case["op"] == "assign":
        return list(_plain_assign(case, x))
    return _plain_step(case, state, x)


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _plain_assign(case, x):
    page, seqs = case["page"], case["seqs"]
    rows = sum(_sizes(case)[1]) + case["pad"]
    tables, free, n_free = x["tables"].clone(), x["free"], x["n_free"].long()
    lens, new = x["lens"].long(), x["new"].long()
    width = tables.shape[1]

    def pages_of(n):
        return (n + page - 1).div(page, rounding_mode="floor")

    need = pages_of(lens + new) - pages_of(lens)
    status = (need.sum() > n_free).long() + 2 * (pages_of(lens + new) > width).any() + 4 * (new.sum() > rows) + 8 * ((lens < 0).any() | (new < 0).any())
    new = torch.where(status == 0, new, 0)
    need = torch.where(status == 0, need, 0)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), new.cumsum(0)))
    token = torch.arange(rows, device="cuda")
    there = token < cu[-1]
    seq = torch.searchsorted(cu[1:], token, right=True).clamp_max(seqs - 1)
    position = torch.where(there, lens[seq] + token - cu[seq], 0)
    column = position // page
    lacking = column - pages_of(lens)[seq]
    taken = n_free - 1 - (need.cumsum(0) - need)[seq] - lacking
    number = torch.where(lacking < 0, tables[seq, column].long(), free[taken.clamp(0, free.numel() - 1)].long())
    # (tokens that are not there write what is there into the last entry of the last row)
    at = torch.where(there, seq * width + column, seqs * width - 1)
    flat = tables.view(-1)
    flat[at] = torch.where(there, number.to(torch.int32), flat[-1])
    slots = torch.where(there, number * page + position % page, -1)
    return (tables, (lens + new).to(torch.int32), cu.to(torch.int32), slots, torch.where(there, position, -1).to(torch.int32),
            (n_free - need.sum()).to(torch.int32), status.to(torch.int32))


def _plain_step(case, state, x):
    hq, hkv, d, page = (case[k] for k in ("hq", "hkv", "d", "page"))
    pages, total = (x["k_pages"], x["v_pages"]), sum(state["new"])
    out, lse = state["out"], state["lse"]
    slots = x["slots"][:total]
    for held, new in zip(pages, (x["k"], x["v"])):
        held[slots // page, :, slots % page] = new[:total]
    first = 0
    for s, (prev, n) in enumerate(zip(state["prev"], state["new"])):
        if n == 0:
            continue
        length = prev + n
        table = x["tables"][s, :-(-length // page)].long()
        keys, values = (held[table].transpose(0, 1).reshape(hkv, -1, d)[:, :length].float() for held in pages)
        across = keys.transpose(1, 2).contiguous()
        block = max(1, 2 ** 30 // (hq * length))
        for i in range(0, n, block):
            m = min(block, n - i)
            rows = x["q"][first + i:first + i + m].float().view(m, hkv, hq // hkv, d).transpose(0, 1).reshape(hkv, -1, d)
            p = torch.bmm(rows, across).mul_(1.0 / math.sqrt(d))
            later = torch.arange(length, device="cuda")[None, :] > torch.arange(prev + i, prev + i + m, device="cuda")[:, None]
            p.view(hkv, m, hq // hkv, length).masked_fill_(later[None, :, None, :], -math.inf)
            top = p.amax(-1, keepdim=True)
            p.sub_(top).exp_()
            sums = p.sum(-1, keepdim=True)
            o = torch.bmm(p, values).div_(sums)
            out[first + i:first + i + m] = o.view(hkv, m, hq // hkv, d).transpose(0, 1).reshape(m, hq, d).to(out.dtype)
            lse[:, first + i:first + i + m] = (top + sums.log()).view(hkv, m, hq // hkv).transpose(1, 2).reshape(hq, m)
        first += n
    return {"out": out, "lse": lse, "pages": pages}


# ---- 64 bits, by the definitions ----------------------------------------------------------------------------------------
def exact(case, seed):
    prev, new = _sizes(case)
    page, hq, hkv, d = (case[k] for k in ("page", "hq", "hkv", "d"))
    rows, group = sum(new) + case["pad"], hq // hkv
    if case["op"] == "assign":
        x = _pages(case, _generator(seed))
        tables, free, n_free = x["tables"].tolist(), x["free"].tolist(), x["n_free"]
        lacking = sum(-(-(p + n) // page) + (-p // page) for p, n in zip(prev, new))
        status = 1 if lacking > n_free else 0  # (rows of the table, and places, are enough here)
        cu, places, positions, lens = [0], [], [], []
        for s, (p, n) in enumerate(zip(prev, new)):
            n = 0 if status else n
            for at in range(p, p + n):
                if at % page == 0:
                    n_free -= 1
                    tables[s][at // page] = free[n_free]
                places.append(tables[s][at // page] * page + at % page)
                positions.append(at)
            cu.append(cu[-1] + n)
            lens.append(p + n)
        for more in (places, positions):
            more.extend([-1] * (rows - len(more)))
        as_int = [torch.tensor(v, dtype=t, device="cuda") for v, t in ((tables, torch.int32), (lens, torch.int32), (cu, torch.int32), (places, torch.int64),
                                                                     (positions, torch.int32), ([n_free], torch.int32))]
        return as_int + [torch.tensor([status], dtype=torch.int32, device="cuda")]
    x = _inputs(case, seed)
    held = [x["k_pages"], x["v_pages"]]
    out = torch.zeros((rows, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((hq, rows), dtype=torch.float64, device="cuda")
    first = 0
    for s, (p, n) in enumerate(zip(prev, new)):
        at = torch.arange(p + n, device="cuda")
        numbers = x["tables"][s].long()[at // page]
        for pages, more in zip(held, (x["k"], x["v"])):
            pages[numbers[p:], :, at[p:] % page] = more[first:first + n]
        if n:
            k, v = (pages[numbers, :, at % page].double() for pages in held)
            step = max(1, 2 ** 27 // (p + n))
            for h in range(hq):
                for i in range(0, n, step):
                    q = x["q"][first + i:min(first + n, first + i + step), h].double()
                    s64 = q @ k[:, h // group].T / math.sqrt(d)
                    seen = at[None, :] <= p + i + torch.arange(q.shape[0], device="cuda")[:, None]
                    s64 = torch.where(seen, s64, -math.inf)
                    lse[h, first + i:first + i + q.shape[0]] = torch.logsumexp(s64, -1)
                    out[first + i:first + i + q.shape[0], h] = torch.softmax(s64, -1) @ v[:, h // group]
        first += n
    return {"out": out, "lse": lse, "pages": tuple(held)}
