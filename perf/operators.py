"""The operators of a decoder's attention block, as cases that can be timed and compared.

A decoder that answers token by token spends its step on three things, and these are the operators measured here:

* "linear": a product in 8-bit integers.  The activations are quantised row by row (one scale for each token), multiplied with weights that were
  quantised once (one scale for each output channel), and the epilogue gives back fp16: bias, GELU and a residual among it.
* "append": the keys and values of a step's new tokens go into a paged cache, rotated by their positions on the way, and the queries are rotated with
  them.  The cache holds fp16, or 8-bit integers with a scale for each page and head, which grows with the page's largest value.
* "attend": attention of the new tokens over that cache, causal, optionally with a sliding window and a few first tokens that stay visible.

A batch is what a server forms: sequences of different lengths, a number of new tokens for each, and pages scattered over the cache.  Lengths follow
from the case; what the tensors hold comes from the seed.  Pages and scales of an 8-bit cache are returned as the cache holds them: they are whole
numbers and have to be equal, the order of every operation on the way to them being part of the operator's definition.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"


# ---- the cases ---------------------------------------------------------------------------------------------------

def _linear(name, rows, inner, cols, act="none", res=False):
    return {"name": name, "op": "linear", "rows": rows, "inner": inner, "cols": cols, "act": act, "res": res}


def _append(name, seqs, new, past, kv_heads, group, head_dim, page, cache, rotated, interleaved=False):
    return {"name": name, "op": "append", "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1],
            "kv_heads": kv_heads, "group": group, "head_dim": head_dim, "page": page, "cache": cache, "rotated": rotated, "interleaved": interleaved}


def _attend(name, seqs, new, past, kv_heads, group, head_dim, page, cache, window=0, sinks=0):
    return {"name": name, "op": "attend", "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "past_lo": past[0], "past_hi": past[1],
            "kv_heads": kv_heads, "group": group, "head_dim": head_dim, "page": page, "cache": cache, "window": window, "sinks": sinks}


def listed():
    return [
        # one client, one token: the output projection of a decode step, bound by 16 MB of weights and by latency
        _linear("linear_token", 1, 4096, 4096),
        # a decode step of 48 clients: the widening product of a feed-forward block, still bound by its weights
        _linear("linear_decode", 48, 4096, 16384, act="gelu"),
        # a chunk of one prompt in sizes that fill no tile, with the residual that a block adds
        _linear("linear_ragged", 509, 2064, 5003, res=True),
        # prompts of a full batch: bound by the matrix pipes
        _linear("linear_prompts", 8192, 4096, 16384),
        # a step of 128 clients into a cache of 8-bit integers: each touches one page of every head; latency
        _append("append_decode_int8", 128, (1, 1), (1, 700), 8, 4, 128, 64, "int8", 128),
        # prompts' chunks of any length, on top of what is there: pages that are continued, filled and begun
        _append("append_chunks_int8", 9, (1, 900), (0, 1500), 8, 4, 128, 64, "int8", 128),
        # whole prompts at once into fp16, half of each head rotated, neighbours in pairs
        _append("append_prompts_fp16", 6, (700, 2048), (0, 0), 16, 1, 64, 32, "fp16", 32, True),
        # one client with a conversation of a few thousand tokens behind it: latency, and one sequence's cache shared out over the chip
        _attend("attend_token_int8", 1, (1, 1), (4100, 4100), 8, 4, 128, 64, "int8"),
        # a step of 32 clients of up to 16 thousand tokens: bound by the cache's bytes
        _attend("attend_decode_int8", 32, (1, 1), (1000, 16383), 8, 4, 128, 64, "int8"),
        # long streams: 65 thousand tokens each, of which the last 4096 and the first 4 are seen; fp16
        _attend("attend_stream_fp16", 24, (1, 1), (60000, 65000), 4, 8, 128, 32, "fp16", 4096, 4),
        # chunks of four prompts, some with a past: bound by the matrix pipes
        _attend("attend_chunk_int8", 4, (1200, 2048), (0, 2048), 8, 4, 128, 64, "int8"),
        # a chunk of prompts where each token sees a window and the first tokens, smaller heads, a kv head for each
        _attend("attend_window_fp16", 5, (333, 4001), (0, 300), 12, 1, 64, 128, "fp16", 1024, 16),
    ]


def _spread(n, lo, hi, turn):
    """n whole numbers between lo and hi, spread over the range in no order; the same ones each time."""
    return [lo + int((hi - lo + 1) * ((0.5 + (i + turn) * 0.6180339887498949) % 1.0)) if hi > lo else lo for i in range(n)]


def _lengths(case):
    new = _spread(case["seqs"], case["new_lo"], case["new_hi"], 0)
    past = _spread(case["seqs"], case["past_lo"], case["past_hi"], 7)
    return new, [a + b for a, b in zip(past, new)]


def _between(rng, lo, hi):
    return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    most = {(c["op"], what): max(work(d)[what] for d in listed() if d["op"] == c["op"]) for c in listed() for what in ("flops", "bytes")}
    while True:
        op = rng.choice(("linear", "append", "attend", "attend"))
        if op == "linear":
            case = _linear("", _between(rng, 1, 8192), 16 * _between(rng, 4, 512), _between(rng, 64, 16384), rng.choice(("none", "none", "gelu", "relu")), rng.random() < 0.4)
        else:
            chunk = rng.random() < 0.5
            seqs = _between(rng, 1, 8 if chunk else 128)
            new = _between(rng, 2, 2048) if chunk else 1
            past = _between(rng, 1, 16384) if rng.random() < 0.8 else 0
            common = (seqs, (1 + new // 3, new), (past // 5, past), rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 7, 8)), rng.choice((64, 128)), rng.choice((32, 64, 128)),
                      rng.choice(("int8", "int8", "fp16")))
            if op == "append":
                case = _append("", *common, rotated=rng.choice((16, 32, 64)) if common[5] == 64 or rng.random() < 0.3 else 128, interleaved=rng.random() < 0.4)
            else:
                window = _between(rng, 16, 4096) if rng.random() < 0.5 else 0
                case = _attend("", *common, window=window, sinks=rng.choice((0, 1, 4, 40)) if window else 0)
        w = work(case)
        # (what the plain form holds at once is bounded as well: all scores, or the whole cache in 32 bits)
        if w["flops"] <= most[op, "flops"] and w["bytes"] <= most[op, "bytes"] and _plain_size(case) <= 2 ** 31:
            del case["name"]
            return case


def _plain_size(case):
    if case["op"] == "linear":
        return case["rows"] * case["cols"]
    new, total = _lengths(case)
    seen = min(max(total), case["window"] + case["sinks"] + max(new)) if case["op"] == "attend" and case["window"] else max(total)
    keys = case["seqs"] * seen * case["kv_heads"] * case["head_dim"]
    return max(keys, case["seqs"] * max(new) * seen * case["kv_heads"] * case["group"]) if case["op"] == "attend" else keys


def _visible(n, total, window, sinks):
    """Of n queries at the end of `total` tokens: visible (query, key) pairs, and the keys that any of them sees."""
    p = np.arange(total - n, total, dtype=np.int64)
    if not window:
        return int((p + 1).sum()), total
    first = np.maximum(p - window + 1, 0)
    pairs = int((p - first + 1 + np.minimum(first, sinks)).sum())
    return pairs, int(total - first[0] + min(first[0], sinks))


def work(case):
    if case["op"] == "linear":
        m, k, n = case["rows"], case["inner"], case["cols"]
        return {"bytes": 2 * m * k + n * k + 8 * n + 2 * m * n * (2 if case["res"] else 1), "flops": 2 * m * n * k}
    new, total = _lengths(case)
    hkv, d, size = case["kv_heads"], case["head_dim"], 1 if case["cache"] == "int8" else 2
    hq, tokens = hkv * case["group"], sum(new)
    if case["op"] == "append":
        return {"bytes": tokens * ((hq + 2 * hkv) * d * 2 + hq * d * 2 + 2 * hkv * d * size + case["rotated"] * 4),
                "flops": tokens * (hq + hkv) * case["rotated"] * 3}
    seen = [_visible(n, t, case["window"], case["sinks"]) for n, t in zip(new, total)]
    return {"bytes": sum(keys for _, keys in seen) * 2 * hkv * d * size + tokens * hq * d * 4, "flops": 4 * d * hq * sum(pairs for pairs, _ in seen)}


# ---- what a program has in hand --------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7fffffffffff)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float16)


def _codes(g, *shape):
    return _normal(g, *shape).mul_(36).clamp_(-127, 127).round_().to(torch.int8)


def _scales(g, *shape):
    return torch.randn(shape, generator=g, device=DEV).mul_(0.25).exp_().mul_(0.03)


def _prepare_linear(case, g):
    m, k, n = case["rows"], case["inner"], case["cols"]
    return {"x": _normal(g, m, k), "w": _codes(g, n, k), "w_scale": _scales(g, n) / k ** 0.5, "bias": torch.randn(n, generator=g, device=DEV) * 0.1,
            "res": _normal(g, m, n) if case["res"] else None}


def _prepare_cached(case, g):
    new, total = _lengths(case)
    hkv, d, page = case["kv_heads"], case["head_dim"], case["page"]
    hq, tokens, seqs = hkv * case["group"], sum(new), case["seqs"]
    each = [-(-t // page) for t in total]
    pages = sum(each) + 3
    s = {"new": max(new), "longest": max(total), "seqs": seqs}
    # the sequences' pages lie anywhere in the cache
    order = torch.randperm(pages, generator=g, device=DEV)[:sum(each)].to(torch.int32)
    width = max(each)
    column = torch.arange(width, device=DEV)[None, :]
    has = column < torch.tensor(each, device=DEV)[:, None]
    s["table"] = torch.full((seqs, width), -1, dtype=torch.int32, device=DEV)
    s["table"][has] = order
    s["q_start"] = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
    s["kv_len"] = torch.tensor(total, dtype=torch.int32, device=DEV)
    shape = (pages, hkv, page, d)
    if case["cache"] == "int8":
        s["k"], s["v"], s["k_scale"], s["v_scale"] = _codes(g, *shape), _codes(g, *shape), _scales(g, pages, hkv), _scales(g, pages, hkv)
    else:
        s["k"], s["v"], s["k_scale"], s["v_scale"] = _normal(g, *shape), _normal(g, *shape), None, None
    if case["op"] == "append":
        qkv = _normal(g, tokens, (hq + 2 * hkv) * d)                # as the product in front leaves it
        s["qkv"] = qkv
        r = case["rotated"]
        angle = torch.arange(max(total), dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
        s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV)
    else:
        s["q"] = _normal(g, tokens, hq * d) * 2
    return s


def prepare(case, seed):
    g = _generator(seed)
    s = _prepare_linear(case, g) if case["op"] == "linear" else _prepare_cached(case, g)
    s["case"] = case
    if own:
        import paper_2604_28175_amd as strait
        s["strait"] = strait
        if case["op"] == "linear":
            s["act_code"] = {"none": strait.ACT_NONE, "relu": strait.ACT_RELU, "gelu": strait.ACT_GELU}[case["act"]]
        else:                                                        # the handles that a serving program keeps
            s["cache"] = strait.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
            s["batch"] = strait.KvBatch(s["q_start"], s["kv_len"], s["table"], max_q=s["new"], max_kv=s["longest"])
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    if own:
        return {"linear": _own_linear, "append": _own_append, "attend": _own_attend}[case["op"]](s, case)
    return {"linear": _plain_linear, "append": _plain_append, "attend": _plain_attend}[case["op"]](s, case)


def _own_linear(s, case):
    strait = s["strait"]
    codes, scale = strait.k_quantize_rows(s["x"])
    return strait.k_gemm_i8(codes, scale, s["w"], s["w_scale"], s["bias"], act=s["act_code"], res=s["res"])


def _heads(s, case):
    """The fused projection's columns of q, k and v."""
    hq, hkv, d = case["kv_heads"] * case["group"], case["kv_heads"], case["head_dim"]
    return s["qkv"][:, :hq * d], s["qkv"][:, hq * d:(hq + hkv) * d], s["qkv"][:, (hq + hkv) * d:]


def _own_append(s, case):
    q, k, v = _heads(s, case)
    out = {"q": s["strait"].k_kv_append(s["cache"], s["batch"], k, v, q=q, rope=s["rope"], interleaved=case["interleaved"]), "k": s["k"], "v": s["v"]}
    return out if s["k_scale"] is None else {**out, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _own_attend(s, case):
    return s["strait"].k_attention_paged(s["q"], s["cache"], s["batch"], case["head_dim"] ** -0.5, window=case["window"], sinks=case["sinks"])


def _plain_linear(s, case):
    x = s["x"].float()
    scale = x.abs().amax(1) / 127.0
    codes = torch.round(x * torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))[:, None])
    y = torch.matmul(codes, s["w"].float().t()) * (scale[:, None] * s["w_scale"][None, :]) + s["bias"]
    if s["res"] is not None:
        y = y + s["res"].float()
    if case["act"] == "relu":
        y = y.clamp_min(0)
    if case["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * 0.5 ** 0.5))
    return y.half()


def _places(s):
    """Of each new token: its sequence and its position."""
    t = torch.arange(s["tokens"], device=DEV)
    b = torch.searchsorted(s["q_start"][1:].long(), t, right=True)
    return b, s["kv_len"].long()[b] - s["q_start"].long()[b + 1] + t


def _rotate(x, rope, case):
    r = case["rotated"]
    c, n = rope[:, None, :r // 2], rope[:, None, r // 2:]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * c - b * n, b * c + a * n
    turned = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_append(s, case):
    hkv, d, page = case["kv_heads"], case["head_dim"], case["page"]
    q, k, v = (x.float().unflatten(1, (-1, d)) for x in _heads(s, case))
    s["tokens"] = q.shape[0]
    b, p = _places(s)
    at, row = s["table"].long()[b, p // page], p % page
    rope = s["rope"][p]
    q, k = _rotate(q, rope, case), _rotate(k, rope, case)
    out = {"q": q.half().flatten(1), "k": s["k"], "v": s["v"]}
    if case["cache"] == "fp16":
        s["k"][at, :, row], s["v"][at, :, row] = k.half(), v.half()
        return out
    # a sequence's first page of this call may hold older tokens, whose codes follow the page's scale where that grows
    first = s["kv_len"].long() - (s["q_start"][1:] - s["q_start"][:-1]).long()
    head, old = s["table"].long()[torch.arange(s["seqs"], device=DEV), first // page], first % page
    for x, codes, scale in ((k, s["k"], s["k_scale"]), (v, s["v"], s["v_scale"])):
        before = scale.clone()
        before[at[row == 0]] = 0
        largest = torch.zeros_like(scale).scatter_reduce_(0, at[:, None].expand(-1, hkv), x.abs().amax(2), "amax")
        now = torch.maximum(before, largest / 127.0)
        factor = before / torch.where(now > 0, now, torch.ones_like(now))
        touched = codes[head]
        older = torch.arange(page, device=DEV)[None, None, :, None] < old[:, None, None, None]
        grown = (now > before)[head][:, :, None, None]
        codes[head] = torch.where(older & grown, torch.round(touched.float() * factor[head][:, :, None, None]).to(torch.int8), touched)
        inverse = torch.where(now > 0, 1.0 / now, torch.zeros_like(now))
        codes[at, :, row] = torch.round(x * inverse[at][:, :, None]).to(torch.int8)
        scale[at] = now[at]
    return {**out, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_attend(s, case):
    hkv, d, page, group, seqs = case["kv_heads"], case["head_dim"], case["page"], case["group"], s["seqs"]
    window, sinks = case["window"], case["sinks"]
    n, start, total = s["new"], s["q_start"].long(), s["kv_len"].long()
    count = start[1:] - start[:-1]
    i = torch.arange(n, device=DEV)[None, :]
    real = i < count[:, None]
    rows = (start[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().view(seqs, n, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, group * n, d)
    place = (total - count)[:, None] + i                                                         # of each query
    if window and s["longest"] > window + sinks + n:                                            # the first keys, and those from the first query's window on
        begin = ((total - count) - window + 1).clamp(min=sinks)
        j = torch.cat([torch.arange(sinks, device=DEV)[None, :].expand(seqs, -1), begin[:, None] + torch.arange(window + n, device=DEV)[None, :]], 1)
    else:
        j = torch.arange(s["longest"], device=DEV)[None, :].expand(seqs, -1)
    there = j < total[:, None]
    at = torch.gather(s["table"].long(), 1, (j // page).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    k, v = (x[at, :, j % page].float() for x in (s["k"], s["v"]))                                # [seqs][keys][kv heads][d]
    if case["cache"] == "int8":
        k, v = k * s["k_scale"][at][..., None], v * s["v_scale"][at][..., None]
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    score = torch.matmul(q, k).view(seqs, hkv, group, n, -1) * d ** -0.5
    seen = there[:, None, :] & real[:, :, None] & (j[:, None, :] <= place[:, :, None])
    if window:
        seen = seen & ((place[:, :, None] - j[:, None, :] < window) | (j[:, None, :] < sinks))
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total_p = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).view(seqs, hkv, group, n, d) / torch.where(total_p > 0, total_p, torch.ones_like(total_p))
    return o.permute(0, 3, 1, 2, 4).reshape(seqs, n, hkv * group * d)[real].half()


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def _exact_linear(s, case):
    outs = []
    w = s["w"].double()
    for lo in range(0, case["rows"], 1024):
        x = s["x"][lo:lo + 1024].double()
        step = x.abs().max(1, keepdim=True).values / 127
        whole = (x / step).nan_to_num(0).round()
        y = (whole @ w.mT) * step * s["w_scale"].double() + s["bias"].double()
        y = y + s["res"][lo:lo + 1024].double() if case["res"] else y
        y = y.relu() if case["act"] == "relu" else 0.5 * y * torch.special.erfc(-y / math.sqrt(2)) if case["act"] == "gelu" else y
        outs.append(y)
    return torch.cat(outs)


def _exact_turn(x, position, case):
    """x [heads][d] of one sequence's token range [n] as complex numbers, turned."""
    r = case["rotated"]
    angle = position.double()[:, None] * torch.exp(torch.arange(0, r, 2, device=x.device).double() * (-math.log(10000.0) / r))
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
    y = x.clone()
    if case["interleaved"]:
        z = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) * turn
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    else:
        h = r // 2
        z = torch.complex(x[..., :h], x[..., h:r]) * turn
        y[..., :h], y[..., h:r] = z.real, z.imag
    return y


def _exact_append(s, case):
    hkv, d, page = case["kv_heads"], case["head_dim"], case["page"]
    hq = hkv * case["group"]
    new, total = _lengths(case)
    qs, cache = [], {"k": s["k"].double(), "v": s["v"].double()}
    scale = {"k": s["k_scale"].double(), "v": s["v_scale"].double()} if case["cache"] == "int8" else None
    base = 0
    for b, (n, t) in enumerate(zip(new, total)):
        x = s["qkv"][base:base + n].double().view(n, -1, d)
        base += n
        position = torch.arange(t - n, t, device=DEV)
        qs.append(_exact_turn(x[:, :hq], position, case).flatten(1))
        parts = {"k": _exact_turn(x[:, hq:hq + hkv], position, case), "v": x[:, hq + hkv:]}
        for c in range((t - n) // page, (t - 1) // page + 1):
            g = int(s["table"][b, c])
            lo, hi = max(t - n, c * page), min(t, (c + 1) * page)
            for name, y in parts.items():
                y = y[lo - (t - n):hi - (t - n)].transpose(0, 1)                # [kv heads][tokens][d]
                if scale is None:
                    cache[name][g, :, lo - c * page:hi - c * page] = y
                    continue
                before = scale[name][g] if lo > c * page else torch.zeros(hkv, device=DEV, dtype=torch.float64)
                scale[name][g] = torch.maximum(before, y.abs().amax((1, 2)) / 127)
    q = torch.cat(qs)
    if scale is None:
        return {"q": q, "k": cache["k"], "v": cache["v"]}
    return {"q": q, "k": None, "v": None, "k_scale": scale["k"], "v_scale": scale["v"]}         # (whole numbers are compared as they are)


def _exact_attend(s, case):
    hkv, d, page, group = case["kv_heads"], case["head_dim"], case["page"], case["group"]
    new, total = _lengths(case)
    outs, base = [], 0
    for b, (n, t) in enumerate(zip(new, total)):
        pages = s["table"][b, :-(-t // page)].long()
        k, v = s["k"][pages].double(), s["v"][pages].double()                  # [pages][kv heads][page][d]
        if case["cache"] == "int8":
            k, v = k * s["k_scale"][pages].double()[..., None, None], v * s["v_scale"][pages].double()[..., None, None]
        k, v = k.transpose(0, 1).flatten(1, 2)[:, :t], v.transpose(0, 1).flatten(1, 2)[:, :t]
        q = s["q"][base:base + n].double().view(n, hkv, group, d)
        base += n
        at = torch.arange(t - n, t, device=DEV)[:, None] - torch.arange(t, device=DEV)[None, :]
        seen = at >= 0
        if case["window"]:
            seen = seen & ((at < case["window"]) | (torch.arange(t, device=DEV)[None, :] < case["sinks"]))
        o = torch.empty(n, hkv, group, d, device=DEV, dtype=torch.float64)
        for h in range(hkv):
            for g in range(group):
                score = (q[:, h, g] @ k[h].mT) / math.sqrt(d)
                o[:, h, g] = score.masked_fill(~seen, -math.inf).softmax(-1) @ v[h]
        outs.append(o.flatten(1))
    return torch.cat(outs)


def exact(case, seed):
    g = _generator(seed)
    if case["op"] == "linear":
        return _exact_linear(_prepare_linear(case, g), case)
    s = _prepare_cached(case, g)
    return _exact_append(s, case) if case["op"] == "append" else _exact_attend(s, case)
