"""Operators that make a carried cache smaller, as measurable cases.

Three operators, each reached through the package's public entry points:

* "step": a fold step on a cache that is held in 8 bits (`KvFoldQuantCache.step`).  Block b of a KV head, its rows 64 b ... 64 b + 63, is
  held as whole numbers of -127 ... 127 and one scale each for K and V as soon as all its rows are there:
      scale = max(max |x| / 127, 2^-100),   code = x / scale rounded to the nearest whole number (ties to even),
  quotients rounded to 32 bits.  Rows of the last, incomplete block are held as they came (bf16).  The chunk's rows are appended first; query
  row i, at position prev + i, then attends to every row j <= prev + i as the cache holds it.
* "weigh": the softmax weight that a step's queries gave to each cached key, summed over the chunk's rows and the query heads of the KV
  head's group (`KvFoldCache.weigh`): w[g][j] = sum over i, h of exp(scale q[i][h] . k[g][j] - lse[h][i]), j <= prev + i.
* "evict": the rows of a layer that are kept -- the first `sink`, the last `recent` and, between them, those with the largest weights, equal
  weights by the lowest index -- moved in their order to another cache (`KvFoldCache.evict`).

Keys of a case: op, dtype ("bf16" or "f32"), hq / hkv / d (query heads, KV heads, head dim), n (the chunk's tokens), prev (tokens in the cache before
them), rope (the step rotates q and k), add (weigh: onto weights that are there), keep / sink / recent (evict; prev is then the cache's whole length).
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 64            # rows that share a scale
LEAST_SCALE = 2.0 ** -100
_MAX_TOKENS = 131072


def _case(name, op, dtype="bf16", hq=32, hkv=8, d=128, n=1, prev=0, rope=False, add=False, keep=0, sink=0, recent=0):
    case = {"name": name, "op": op, "dtype": dtype, "hq": hq, "hkv": hkv, "d": d, "n": n, "prev": prev, "rope": rope, "add": add, "keep": keep,
            "sink": sink, "recent": recent}
    if name is None:
        del case["name"]
    return case


def listed():
    return [
        # The smallest call: one token after a short prompt, Llama-3.1-8B heads.
        _case("step_decode_300", "step", n=1, prev=300),
        # Greedy decoding after a short document of no round length.
        _case("step_decode_4k", "step", n=1, prev=4187),
        # Greedy decoding after the long chain: bound by reading the cache.
        _case("step_decode_128k", "step", n=1, prev=130941),
        # The question behind the document, with a length of its own and the rotary embedding inside the step.
        _case("step_question_rope_32k", "step", n=37, prev=32768, rope=True),
        # One step of the deep chain of 256-token chunks, half way.
        _case("step_chain_c256_64k", "step", n=256, prev=65536),
        # A prefill chunk of the 128K workload's heads, at 32K; the largest case.
        _case("step_c2048_32k", "step", n=2048, prev=32768),
        # A model with 64-wide heads, chunks off any grid.
        _case("step_d64_c1000_8k", "step", d=64, n=1000, prev=8192),
        # Weights of one decoding step, added to those so far.
        _case("weigh_decode_16k", "weigh", n=1, prev=16301, add=True),
        # Weights of a whole chunk of the deep chain (28 query heads on 4, the sweep's), without a history.
        _case("weigh_c256_64k", "weigh", hq=28, hkv=4, n=256, prev=65536),
        # The smallest workload of the fold, in fp32.
        _case("weigh_tiny_f32", "weigh", dtype="f32", hq=4, hkv=1, d=64, n=128, prev=384, add=True),
        # Serving with a budget: a cache that outgrew its 1024 tokens by a chunk.
        _case("evict_1280_to_1024", "evict", prev=1280, keep=1024, sink=4, recent=256),
        # A long document's cache halved before decoding.
        _case("evict_128k_to_64k", "evict", prev=130941, keep=65536, sink=4, recent=1020),
    ]


# Head shapes of the repository's configurations and tests: (query heads, KV heads, head dim).
_SHAPES = ((32, 8, 128), (32, 8, 128), (28, 4, 128), (32, 8, 64), (4, 1, 64), (8, 2, 128))


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(case):
    """Rough seconds of a pass, for keeping drawn cases no larger than the largest listed one."""
    w = work(case)
    return max(w["flops"] / (1e15 if case["dtype"] == "bf16" else 1e14), w["bytes"] / 5e12)


def draw(rng):
    limit = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("step", "step", "weigh", "evict"))
        hq, hkv, d = rng.choice(_SHAPES)
        case = dict(hq=hq, hkv=hkv, d=d)
        prev = _log_uniform(rng, 16, _MAX_TOKENS)
        if op == "step":
            n = rng.choice((1, 1, rng.randint(2, 16), rng.randint(17, 64), _log_uniform(rng, 65, 2048)))
            # (a pass goes back to where it began: any place for short steps, a block's beginning for long ones)
            case.update(n=n, prev=prev if n <= BLOCK else prev // BLOCK * BLOCK, rope=rng.random() < 0.25)
        elif op == "weigh":
            case.update(n=rng.choice((1, _log_uniform(rng, 2, 1024))), prev=prev, add=rng.random() < 0.5, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
        else:
            sink, recent = rng.choice((0, 4, 16)), rng.choice((0, 32, 1020))
            least = max(1, sink + recent)
            case.update(prev=prev, sink=sink, recent=recent, keep=_log_uniform(rng, least, max(least, prev)), dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
        case = _case(None, op, **case)
        if case["prev"] + case["n"] <= _MAX_TOKENS and case["keep"] <= case["prev"] and _cost(case) <= limit:
            return case


def work(case):
    """Step: the codes and scales of the cache, q, the new rows read and written, the output and the log-sum-exp; two products over the visible
    (row, key) pairs.  Weigh: the K rows, q, the log-sum-exps, the weights; one product.  Evict: the weights, and the kept rows read and written."""
    es = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d, n, prev = (case[k] for k in ("hq", "hkv", "d", "n", "prev"))
    pairs = n * (prev + (n + 1) / 2.0)
    angles = 4.0 * n * d if case["rope"] else 0.0
    if case["op"] == "step":
        cached = 2.0 * hkv * d * prev + 8.0 * hkv * (prev // BLOCK)
        return {"bytes": cached + 2.0 * hkv * d * n * (2 + 1) + 4.0 * n * hq * d + 4.0 * n * hq + angles, "flops": 4.0 * hq * d * pairs}
    if case["op"] == "weigh":
        return {"bytes": float(es) * hkv * d * (prev + n) + float(es) * n * hq * d + 4.0 * n * hq + 4.0 * hkv * (prev + n) * (2 if case["add"] else 1),
                "flops": 2.0 * hq * d * pairs}
    return {"bytes": 4.0 * hkv * (prev + 2 * case["keep"]) + 4.0 * es * hkv * d * case["keep"], "flops": 0.0}


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _inputs(case, seed):
    """Rows, queries and weights of a case, from the seed alone.  Keys have channels of different sizes, as a model's have."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 20260512)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    hq, hkv, d, n, prev = (case[k] for k in ("hq", "hkv", "d", "n", "prev"))
    x = {"gain": torch.exp(0.4 * _normal(gen, hkv, d))}
    x["k_prev"] = (_normal(gen, prev, hkv, d) * x["gain"]).to(dt)
    x["v_prev"] = _normal(gen, prev, hkv, d).to(dt)
    if case["op"] == "evict":
        # sums of softmax weights spread over orders of magnitude; many keys got nothing at all, and equal sums occur
        w = torch.exp(2.0 * _normal(gen, hkv, prev) - 6.0)
        w = torch.where(torch.rand(hkv, prev, generator=gen, device="cuda") < 0.1, torch.zeros_like(w), w)
        x["weights"] = torch.where(torch.rand(hkv, prev, generator=gen, device="cuda") < 0.1, (w * 256).round() / 256, w)
        return x
    x["q"] = _normal(gen, n, hq, d).to(dt)
    x["k"] = (_normal(gen, n, hkv, d) * x["gain"]).to(dt)
    x["v"] = _normal(gen, n, hkv, d).to(dt)
    if case["rope"]:
        at = torch.arange(prev, prev + n, device="cuda", dtype=torch.float64)
        angle = at[:, None] * 500000.0 ** (torch.arange(d // 2, device="cuda", dtype=torch.float64) * (-2.0 / d))
        x["rope"] = (angle.cos().float(), angle.sin().float())
    if case["op"] == "weigh":
        keys = torch.cat((x["k_prev"], x["k"])).transpose(0, 1)
        x["lse"] = torch.logsumexp(_logits(x["q"], keys, prev), dim=-1).view(hkv, n, hq // hkv).transpose(1, 2).reshape(hq, n).contiguous()
        if case["add"]:
            x["weights"] = torch.exp(2.0 * _normal(gen, hkv, prev + n) - 6.0)
    return x


def prepare(case, seed):
    """The inputs, and what holds the cache: the library's, or in the plain form tensors."""
    hq, hkv, d, n, prev, keep = (case[k] for k in ("hq", "hkv", "d", "n", "prev", "keep"))
    x = _inputs(case, seed)
    state = {"case": case, "x": x}
    if case["op"] == "step":
        state["out"] = torch.empty_like(x["q"])
        state["lse"] = torch.empty((hq, n), device="cuda")
        state["first"] = prev - prev % BLOCK if (prev + n) // BLOCK > prev // BLOCK else prev  # the rows that the step adds or changes
        state["rows"] = [torch.empty((prev + n - state["first"], hkv, d), device="cuda") for _ in range(2)]
        if own:
            from paper_2605_12471_amd import KvFoldQuantCache
            cache = KvFoldQuantCache(1, hq, hkv, d, max(n, 256), max(-(-(prev + n) // 1024) * 1024, 1024))
            cache.append(0, x.pop("k_prev"), x.pop("v_prev"))
            state["cache"] = cache
        else:
            whole = prev - prev % BLOCK
            for name in ("k", "v"):
                rows = x.pop(name + "_prev")
                state[name + "_codes"], state[name + "_scales"] = _held(rows[:whole])
                state[name + "_tail"] = rows[whole:].clone()
        return state
    rows = prev + n if case["op"] == "weigh" else prev
    if own:
        from paper_2605_12471_amd import KvFoldCache
        cache = KvFoldCache(1, hq, hkv, d, min(rows, max(n, 256)), rows, case["dtype"])
        k_rows, v_rows = cache.view(0)
        for view, name in ((k_rows, "k"), (v_rows, "v")):
            view[:, :prev].copy_(x[name + "_prev"].transpose(0, 1))
            if case["op"] == "weigh":
                view[:, prev:].copy_(x[name].transpose(0, 1))
        cache.set_length(0, rows)
        state["cache"] = cache
    if case["op"] == "weigh":
        state["weights"] = x["weights"] if case["add"] else torch.empty((hkv, rows), device="cuda")
        if not own:
            state["keys"] = torch.cat((x["k_prev"], x["k"])).transpose(0, 1).contiguous()
    else:
        state["kept"] = torch.empty((hkv, keep), dtype=torch.int32, device="cuda")
        state["weights"] = torch.empty((hkv, keep), device="cuda")
        if own:
            to = KvFoldCache(1, hq, hkv, d, min(keep, 256), keep, case["dtype"])
            state["to"], state["to_rows"] = to, to.view(0)
            for rows in state["to_rows"]:
                rows.owner = to  # the view aliases the cache's memory: whoever holds the rows keeps the cache
        else:
            state["k_rows"], state["v_rows"] = (x[name].transpose(0, 1).contiguous() for name in ("k_prev", "v_prev"))
    del x["k_prev"], x["v_prev"]
    return state


def run(state):
    case, x = state["case"], state["x"]
    if own:
        if case["op"] == "step":
            cache = state["cache"]
            cache.truncate(0, case["prev"])
            cache.step(0, x["q"], x["k"], x["v"], state["out"], lse=state["lse"], rope=x.get("rope"))
            cache.read(0, state["first"], *state["rows"])
            return {"out": state["out"], "lse": state["lse"], "rows": state["rows"]}
        if case["op"] == "weigh":
            weights = state["weights"].clone() if case["add"] else state["weights"]
            return {"weights": state["cache"].weigh(0, x["q"], x["lse"], weights, add=case["add"])}
        state["cache"].evict(0, x["weights"], case["keep"], case["sink"], case["recent"], to=state["to"], to_weights=state["weights"], kept=state["kept"])
        return {"kept": state["kept"], "rows": state["to_rows"], "weights": state["weights"]}
    if case["op"] == "step":
        return _plain_step(case, state, x)
    if case["op"] == "weigh":
        return {"weights": _plain_weigh(case, state, x)}
    return _plain_evict(case, state, x)


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _held(rows):
    """Codes [r][Hkv][d] and scales [blocks][Hkv] of whole blocks of rows.  (Quotients in 64 bits, rounded to the 32 that the operator defines:
    some lie next to a half.)"""
    x = rows.double().view(-1, BLOCK, rows.shape[1], rows.shape[2])
    scales = (x.abs().amax((1, 3)) / 127.0).float().clamp_min(LEAST_SCALE)
    codes = (x / scales[:, None, :, None].double()).float().round().clamp_(-127, 127).to(torch.int8)
    return codes.view(rows.shape), scales


def _values(codes, scales):
    return codes.float() * scales.repeat_interleave(BLOCK, 0)[:, :, None]


def _rotated(x, rope):
    """Half-split pairs: in 32 bits the product with the sine rounded first, the other added to it exactly, then rounded to x's type."""
    lo, up = x.double().chunk(2, -1)
    cos, sin = (t[:, None, :].double() for t in rope)
    first = lo * cos - (up * sin).float().double()
    second = up * cos + (lo * sin).float().double()
    return torch.cat((first, second), -1).float().to(x.dtype)


def _logits(q, keys, prev):
    """[Hkv][n G][L] of q [n][Hq][d] on keys [Hkv][L][d]; -inf where a row does not see the key."""
    n, hq, d = q.shape
    hkv = keys.shape[0]
    rows = q.float().view(n, hkv, hq // hkv, d).transpose(0, 1).reshape(hkv, -1, d)
    s = torch.bmm(rows, keys.float().transpose(1, 2).contiguous()).mul_(1.0 / math.sqrt(d))
    later = torch.arange(prev + n, device=q.device)[None, :] > torch.arange(prev, prev + n, device=q.device)[:, None]
    s.view(hkv, n, hq // hkv, prev + n).masked_fill_(later[None, :, None, :], -math.inf)
    return s


def _plain_step(case, state, x):
    hq, hkv, d, n, prev = (case[k] for k in ("hq", "hkv", "d", "n", "prev"))
    q, new = x["q"], {"k": x["k"], "v": x["v"]}
    if case["rope"]:
        q, new["k"] = _rotated(q, x["rope"]), _rotated(new["k"], x["rope"])

    def rows_of(name):
        rest = torch.cat((state[name + "_tail"], new[name]))
        whole = rest.shape[0] - rest.shape[0] % BLOCK
        return torch.cat((_values(state[name + "_codes"], state[name + "_scales"]), _values(*_held(rest[:whole])), rest[whole:].float()))

    keys, values = rows_of("k"), rows_of("v")
    s = _logits(q, keys.transpose(0, 1), prev)
    top = s.amax(-1, keepdim=True)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    out = torch.bmm(s, values.transpose(0, 1).contiguous()).div_(total)
    out = out.view(hkv, n, hq // hkv, d).transpose(0, 1).reshape(n, hq, d).to(torch.bfloat16)
    lse = (top + total.log()).view(hkv, n, hq // hkv).transpose(1, 2).reshape(hq, n)
    return {"out": out, "lse": lse, "rows": [keys[state["first"]:], values[state["first"]:]]}


def _plain_weigh(case, state, x):
    hq, hkv, n, prev = (case[k] for k in ("hq", "hkv", "n", "prev"))
    s = _logits(x["q"], state["keys"], prev)
    lse = x["lse"].view(hkv, hq // hkv, n).transpose(1, 2).reshape(hkv, -1, 1)
    w = s.sub_(lse).exp_().sum(1)
    return state["weights"] + w if case["add"] else w


def _plain_evict(case, state, x):
    keep, sink, recent, rows = case["keep"], case["sink"], case["recent"], case["prev"]
    w = x["weights"].clone()
    w[:, :sink] = math.inf
    w[:, rows - recent:] = math.inf
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    kept = torch.sort(order[:, :keep], dim=-1).values
    index = kept[:, :, None].expand(-1, -1, case["d"])
    return {"kept": kept.to(torch.int32), "rows": [torch.gather(state["k_rows"], 1, index), torch.gather(state["v_rows"], 1, index)],
            "weights": torch.gather(x["weights"], 1, kept)}


# ---- 64 bits, by the definitions ----------------------------------------------------------------------------------------
def exact(case, seed):
    x = _inputs(case, seed)
    hq, hkv, d, n, prev = (case[k] for k in ("hq", "hkv", "d", "n", "prev"))
    group = hq // hkv
    if case["op"] == "evict":
        kept = []
        for g in range(hkv):
            between = x["weights"][g, case["sink"]:prev - case["recent"]].cpu()
            best = sorted(range(len(between)), key=between.neg().tolist().__getitem__)[:case["keep"] - case["sink"] - case["recent"]]
            kept.append(list(range(case["sink"])) + sorted(case["sink"] + j for j in best) + list(range(prev - case["recent"], prev)))
        kept = torch.tensor(kept, device="cuda")
        heads = torch.arange(hkv, device="cuda")[:, None]
        return {"kept": kept.to(torch.int32), "rows": [x["k_prev"][kept, heads], x["v_prev"][kept, heads]], "weights": x["weights"][heads, kept]}
    q, held = x["q"].double(), []
    if case["op"] == "step":
        for name in ("k", "v"):
            new = x[name]
            if case["rope"] and name == "k":
                new = _turn(new, x["rope"])
            rows = torch.cat((x[name + "_prev"], new)).double()
            whole = (prev + n) // BLOCK * BLOCK
            for b in range(0, whole, 512 * BLOCK):
                part = rows[b:min(whole, b + 512 * BLOCK)].unflatten(0, (-1, BLOCK))
                scale = (part.abs().amax((1, 3), keepdim=True) / 127).float().double().clamp_min(LEAST_SCALE)
                part.copy_((part / scale).float().double().round().clamp(-127, 127) * scale)
            held.append(rows)
        if case["rope"]:
            q = _turn(x["q"], x["rope"]).double()
    else:
        held.append(torch.cat((x["k_prev"], x["k"])).double())
    at = torch.arange(prev, prev + n, device="cuda")
    seen = torch.arange(prev + n, device="cuda")
    out, lse = torch.empty((n, hq, d), dtype=torch.float64, device="cuda"), torch.empty((hq, n), dtype=torch.float64, device="cuda")
    weights = x["weights"].double() if case["add"] else torch.zeros((hkv, prev + n), dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 28 // (prev + n))
    for h in range(hq):
        for i in range(0, n, step):
            s = q[i:i + step, h] @ held[0][:, h // group].T / math.sqrt(d)
            s = torch.where(seen[None, :] <= at[i:i + step, None], s, -math.inf)
            if case["op"] == "weigh":
                weights[h // group] += torch.exp(s - x["lse"][h, i:i + step, None].double()).sum(0)
                continue
            lse[h, i:i + step] = torch.logsumexp(s, -1)
            out[i:i + step, h] = torch.softmax(s, -1) @ held[1][:, h // group]
    if case["op"] == "weigh":
        return {"weights": weights}
    first = prev - prev % BLOCK if (prev + n) // BLOCK > prev // BLOCK else prev
    return {"out": out, "lse": lse, "rows": [held[0][first:], held[1][first:]]}


def _turn(x, rope):
    """x rotated in 64 bits but for the roundings that the rotary step defines."""
    half = x.shape[-1] // 2
    c, s = rope[0].double().unsqueeze(1), rope[1].double().unsqueeze(1)
    a, b = x[..., :half].double(), x[..., half:].double()
    y = torch.empty_like(x)
    y[..., :half] = (a * c - (b * s).float()).float()
    y[..., half:] = (b * c + (a * s).float()).float()
    return y
