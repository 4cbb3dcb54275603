"""Operators of a decode service whose cache stays inside a budget: what each computes, and what is measured of it.

* ``attend``: attention of one new token per sequence over one layer of the paged KV cache, which also adds up, for every
  cached token and KV head, the attention weight that the token has received (``Context.kv_attend``);
* ``evict``: the tokens with the least accumulated weight leave the cache; the others move together, in every layer and KV head
  by its own choice (``Context.kv_evict``);
* ``sample``: one token per row of logits by temperature, top-k, top-p and min-p from a given random number
  (``binding.sample``).

The layout of the cache is that of ``include/harli.h``: chunks of [layer][K or V] blocks, a block of pages, a page of
[KV head][16 token slots][head size].  A tracking record is a pair (fp32 weight, int32 position) per token and KV head, laid
out [layer][page][KV head][slot].
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
PAGE = 16                # tokens per page
BLOCK = 2 << 20          # bytes per block of the pool
VOCABS = (1000, 8000, 32000, 50257, 128256, 152064)
# (query heads, KV heads, head size): the workloads' own, and layouts their tests use
HEADS = ((32, 32, 128), (40, 40, 128), (32, 8, 128), (28, 4, 128), (8, 2, 64), (6, 2, 128), (8, 4, 128), (5, 1, 128))


# --------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the toy layer in fp32 that a first test of an installation runs: launches and latency
        {"name": "attend_tiny_f32", "op": "attend", "dtype": "f32", "n_q": 4, "n_kv": 4, "d": 64, "batch": 4, "dist": "uniform", "length": 96, "cap": 128, "decay": 1.0},
        # a layer of the 7B class, a service with 16 users at 1024 cached tokens each
        {"name": "attend_7b_b16", "op": "attend", "dtype": "bf16", "n_q": 32, "n_kv": 32, "d": 128, "batch": 16, "dist": "const", "length": 1024, "cap": 1024, "decay": 1.0},
        # grouped queries, one user with a long document: the work has to be split over the cache's length
        {"name": "attend_gqa_long_b1", "op": "attend", "dtype": "bf16", "n_q": 32, "n_kv": 8, "d": 128, "batch": 1, "dist": "const", "length": 32001, "cap": 32001, "decay": 0.98},
        # seven query heads per KV head, a full service with uneven lengths
        {"name": "attend_gqa7_b192", "op": "attend", "dtype": "bf16", "n_q": 28, "n_kv": 4, "d": 128, "batch": 192, "dist": "lognormal", "length": 800, "cap": 8192, "decay": 1.0},
        # the toy layer's cache, four sequences cut to half
        {"name": "evict_tiny_f32", "op": "evict", "dtype": "f32", "n_kv": 4, "d": 64, "layers": 1, "batch": 4, "dist": "uniform", "length": 96, "cap": 128, "keep": 0.5, "sink": 4, "recent": 16},
        # the steady state of a service: a page has filled up and one page's worth of tokens leaves, in every layer
        {"name": "evict_page_b16", "op": "evict", "dtype": "bf16", "n_kv": 8, "d": 128, "layers": 8, "batch": 16, "dist": "const", "length": 1040, "cap": 1040, "keep": 1024.0, "sink": 4, "recent": 128},
        # the pool is short: every sequence of a full service gives back half of what it holds
        {"name": "evict_half_b192", "op": "evict", "dtype": "bf16", "n_kv": 4, "d": 128, "layers": 4, "batch": 192, "dist": "lognormal", "length": 800, "cap": 8192, "keep": 0.5, "sink": 4, "recent": 64},
        # a long document cut to an eighth of it, the layers of a stage
        {"name": "evict_long_b2", "op": "evict", "dtype": "bf16", "n_kv": 8, "d": 128, "layers": 8, "batch": 2, "dist": "const", "length": 30003, "cap": 30003, "keep": 0.125, "sink": 4, "recent": 256},
        # a chat with one user
        {"name": "sample_chat_b1", "op": "sample", "batch": 1, "vocab": 32000, "filters": "k", "temperature": 0.8},
        # a small service, each user with settings of its own
        {"name": "sample_mixed_b23", "op": "sample", "batch": 23, "vocab": 128256, "filters": "mixed", "temperature": 0.9},
        # a rollout: the distribution as it is
        {"name": "sample_plain_b128", "op": "sample", "batch": 128, "vocab": 128256, "filters": "none", "temperature": 1.0},
        # a full service with nucleus sampling over the largest vocabulary
        {"name": "sample_nucleus_b256", "op": "sample", "batch": 256, "vocab": 152064, "filters": "p", "temperature": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attend", "evict", "sample"))
    if op == "sample":
        vocab = rng.choice(VOCABS + (_log(rng, 300, 152064),))
        return {"op": op, "batch": _log(rng, 1, 256), "vocab": vocab, "filters": rng.choice(("none", "k", "p", "m", "kp", "mixed")),
                "temperature": round(rng.uniform(0.5, 1.5), 2)}
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    n_q, n_kv, d = rng.choice(((4, 4, 64), (6, 2, 48), (8, 2, 128), (3, 1, 86))) if dtype == "f32" else rng.choice(HEADS)
    batch, length = _log(rng, 1, 200), _log(rng, 2, 16000)
    layers = 1 if op == "attend" else _log(rng, 1, 8)
    # no more tokens than the largest listed case holds bytes for (a cap keeps the tail of uneven lengths in)
    room = 300e6 if op == "attend" else 900e6
    room = min(room, 2e7) if dtype == "f32" else room
    row = 2 * n_kv * d * (4 if dtype == "f32" else 2) * layers
    length = max(2, min(length, int(room / row / batch)))
    batch = max(1, min(batch, int(room / row / length)))
    case = {"op": op, "dtype": dtype, "n_kv": n_kv, "d": d, "batch": batch, "dist": rng.choice(("const", "uniform", "lognormal")),
            "length": length, "cap": 2 * length + 1}
    if op == "attend":
        return {**case, "n_q": n_q, "decay": rng.choice((1.0, 1.0, 0.95, 0.0))}
    return {**case, "layers": layers, "keep": rng.choice((0.25, 0.5, 0.75, round(rng.uniform(0.05, 0.95), 3), float(max(1, length - 16)))),
            "sink": rng.choice((0, 4)), "recent": rng.choice((0, 16, max(1, length // 10)))}


def _lengths(case, seed):
    """Cached tokens of every sequence: the same lengths for every seed, in another order."""
    r = np.random.default_rng(7)
    n, length, cap = case["batch"], case["length"], case["cap"]
    if case["dist"] == "const":
        got = np.full(n, length)
    elif case["dist"] == "uniform":
        got = r.integers(max(1, 2 * length // 3), min(cap, 4 * length // 3 + 1) + 1, n)
    else:
        got = np.exp(r.normal(math.log(length), 0.6, n))
    return np.random.default_rng(seed).permutation(np.clip(got, 1, cap).astype(np.int32))


def _keep(case, lengths):
    """Tokens that each sequence keeps: a share of them, or a number."""
    k = case["keep"]
    return (np.minimum(lengths, k) if k >= 1 else np.maximum(1, np.floor(lengths * k))).astype(np.int32)


def _element(case):
    return 4 if case["dtype"] == "f32" else 2


def prepare(case, seed):
    return _prepare_rows(case, seed) if case["op"] == "sample" else _prepare_cache(case, seed)


# --------------------------------------------------------------------------------------------- the cache of attend and evict
def _prepare_cache(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    n_kv, d, layers, batch = case["n_kv"], case["d"], case.get("layers", 1), case["batch"]
    lengths = _lengths(case, seed)
    pages = -(-lengths // PAGE)
    max_pages, used = int(pages.max()), int(pages.sum())
    row = n_kv * d * _element(case)
    ppb = BLOCK // (PAGE * row)
    chunks = -(-used // ppb)
    slab_bytes = chunks * layers * 2 * BLOCK
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    slab = torch.empty(slab_bytes, dtype=torch.uint8, device=DEV)
    slab.view(dtype).normal_(generator=g)
    # pages in the order a pool hands them out after a while: scattered
    ids = torch.randperm(chunks * ppb, generator=g, device=DEV, dtype=torch.int32)[:used]
    at = torch.from_numpy(np.arange(max_pages)[None, :] < pages[:, None]).to(DEV)
    table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=DEV)
    table[at] = ids
    n = torch.from_numpy(lengths).to(DEV)
    # [chunk][layer][K, V][page of the block][KV head][slot][head size]
    view = torch.as_strided(slab.view(dtype), (chunks, layers, 2, ppb, n_kv, PAGE, d),
                            (layers * 2 * BLOCK // _element(case), 2 * BLOCK // _element(case), BLOCK // _element(case), PAGE * n_kv * d, PAGE * d, d, 1))
    track = torch.zeros(layers, chunks * ppb, n_kv, PAGE, 2, dtype=torch.int32, device=DEV)
    # the weight that a token has gathered: a few tokens most of it, as attention gives it
    weight = torch.empty(layers, chunks * ppb, n_kv, PAGE, device=DEV).log_normal_(-4.0, 2.0, generator=g)
    track[..., 0] = weight.view(torch.int32)
    slot = torch.arange(max_pages * PAGE, dtype=torch.int32, device=DEV).view(max_pages, PAGE)
    track[:, ids.long(), :, :, 1] = slot.expand(batch, max_pages, PAGE)[at][None, :, None, :]
    s = {"case": case, "slab": slab, "view": view, "ppb": ppb, "table": table, "n": n, "longest": int(lengths.max()), "track": track,
         "used": torch.nonzero(at, as_tuple=True), "tokens": torch.arange(max_pages * PAGE, device=DEV)}
    n_q = case.get("n_q", n_kv)
    if case["op"] == "attend":
        s["q"] = torch.empty(batch, n_q, d, device=DEV).normal_(0.0, 2.0, generator=g)
        s["position"] = n + 7
        s["out"] = torch.empty(batch, n_q, d, device=DEV)
    else:
        s["keep"] = torch.from_numpy(_keep(case, lengths)).to(DEV)
        s["fresh"] = track.clone()
        s["left"] = torch.empty_like(n)
    if own:
        # a decode service's own pool and context, with a layer of few weights: these calls read none of them
        from paper_2511_11729_amd import binding as hb
        pool = hb.Pool(slab, slab_bytes, block_bytes=BLOCK, n_layers=layers, kv_row_bytes=row)
        w = torch.zeros(max(n_q * d, 16) * 16, dtype=dtype, device=DEV)
        gain = torch.ones(16, device=DEV)
        lw = dict.fromkeys(("wq", "wk", "wv", "wo", "wg", "wu", "wd"), w) | {"g1": gain, "g2": gain}
        s["ctx"] = hb.Context(pool, n_layers=layers, hidden=16, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=d, ffn=16,
                              dtype=hb.HARLI_F32 if case["dtype"] == "f32" else hb.HARLI_BF16, max_batch=batch,
                              max_seq_len=s["longest"], layers=[lw] * layers)
        if case["op"] == "attend":
            s["workspace"] = torch.empty(s["ctx"].kv_attend_workspace_bytes(batch, s["longest"]), dtype=torch.uint8, device=DEV)
    return s


def _attend(s):
    case, n, table = s["case"], s["n"], s["table"]
    if own:
        s["ctx"].kv_attend(layer=0, batch=case["batch"], q=s["q"], out=s["out"], n_tokens=n, page_table=table, max_pages=table.shape[1],
                           max_kv_len=s["longest"], track=s["track"], decay=case["decay"], position=s["position"], workspace=s["workspace"])
        return {"out": s["out"], "weight": s["track"][..., 0].view(torch.float32), "position": s["track"][..., 1]}
    batch, n_kv, d = case["batch"], case["n_kv"], case["d"]
    group = case["n_q"] // n_kv
    page = table.long().clamp(min=0)
    kv = s["view"][page // s["ppb"], 0, :, page % s["ppb"]].float()              # [batch, page, K or V, KV head, slot, head size]
    k, v = (kv[:, :, i].transpose(1, 2).reshape(batch * n_kv, -1, d) for i in (0, 1))
    q = (s["q"] / math.sqrt(d)).view(batch * n_kv, group, d)
    inside = s["tokens"] < n[:, None]                                            # [batch, token]
    score = torch.bmm(q, k.transpose(1, 2).contiguous()).view(batch, n_kv, group, -1)
    score = score.masked_fill(~inside[:, None, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = torch.bmm(p.view(batch * n_kv, group, -1), v).view(batch, n_kv * group, d)
    # what every token received, added to its record; the newest token's record begins here
    got = p.sum(2).view(batch, n_kv, -1, PAGE).transpose(1, 2)                   # [batch, page, KV head, slot]
    newest = (s["tokens"] == n[:, None] - 1).view(batch, -1, 1, PAGE)
    old = s["track"][0, page, :, :, 0].view(torch.float32)
    weight = got + torch.where(newest, torch.zeros_like(old), old * case["decay"])
    position = torch.where(newest, s["position"].view(-1, 1, 1, 1), s["track"][0, page, :, :, 1])
    b, t = s["used"]                                                             # the pages that hold tokens
    record = torch.stack((weight[b, t].view(torch.int32), position[b, t]), -1)
    record = torch.where(inside.view(batch, -1, 1, PAGE, 1)[b, t], record, s["track"][0, page[b, t]])
    s["track"][0, page[b, t]] = record
    return {"out": out, "weight": s["track"][..., 0].view(torch.float32), "position": s["track"][..., 1]}


def _evict(s):
    case, n, keep, table = s["case"], s["n"], s["keep"], s["table"]
    s["track"].copy_(s["fresh"])                                                 # the weights that the steps since the last pass left
    if own:
        s["ctx"].kv_evict(batch=case["batch"], n_tokens=n, keep=keep, position=n, page_table=table, max_pages=table.shape[1],
                          max_kv_len=s["longest"], sink=case["sink"], recent=case["recent"], track=s["track"], n_left=s["left"])
        return {"cache": s["view"], "weight": s["track"][..., 0].view(torch.float32), "position": s["track"][..., 1], "n_left": s["left"]}
    page = table.long().clamp(min=0)
    record = s["track"][:, page].permute(0, 1, 3, 2, 4, 5).flatten(3, 4)         # [layer, batch, KV head, token, 2]
    weight, position = record[..., 0].contiguous().view(torch.float32), record[..., 1]
    inside = (s["tokens"] < n[:, None])[None, :, None]
    first = (position < case["sink"]) | (position >= n[None, :, None, None] - case["recent"])
    # protected tokens first, then by weight; equal ones by slot; then what is no token
    rank = torch.where(first, math.inf, weight).masked_fill(~inside, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    place = torch.empty_like(order).scatter_(-1, order, s["tokens"].expand(order.shape))
    left = torch.minimum(n, keep)
    stays = (place < left[None, :, None, None]) & inside
    behind = s["tokens"] >= left[:, None]
    hole = ~stays & ~behind[None, :, None] & inside
    mover = stays & behind[None, :, None]
    # holes and movers are as many in every (layer, sequence, KV head); in order of the slots each meets its partner
    layer, b, c, to = torch.nonzero(hole, as_tuple=True)
    _, _, _, of = torch.nonzero(mover, as_tuple=True)
    there, here = page[b, to // PAGE], page[b, of // PAGE]
    s["view"][there // s["ppb"], layer, :, there % s["ppb"], c, to % PAGE] = s["view"][here // s["ppb"], layer, :, here % s["ppb"], c, of % PAGE]
    s["track"][layer, there, c, to % PAGE] = s["track"][layer, here, c, of % PAGE]
    return {"cache": s["view"], "weight": s["track"][..., 0].view(torch.float32), "position": s["track"][..., 1], "n_left": left}


# --------------------------------------------------------------------------------------------- rows of logits
def _prepare_rows(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    batch, vocab, filters = case["batch"], case["vocab"], case["filters"]
    # a language model's logits: a broad body with a few likely tokens above it, and in every eighth row a mask of a grammar
    logits = torch.empty(batch, vocab, device=DEV).normal_(0.0, 2.5, generator=g)
    peaks = torch.randint(vocab, (batch, 40), device=DEV, generator=g)
    logits.scatter_(1, peaks, torch.empty(batch, 40, device=DEV).normal_(11.0, 2.0, generator=g))
    masked = torch.rand(batch, vocab, device=DEV, generator=g) < 0.5
    masked[torch.arange(batch, device=DEV) % 8 != 7] = False
    logits.masked_fill_(masked, -math.inf)
    r = np.random.default_rng(seed)
    on = np.array([[filters in ("k", "kp"), filters in ("p", "kp"), filters == "m"]] * batch)
    if filters == "mixed":
        on = r.random((batch, 3)) < 0.5
    t = case["temperature"] * r.uniform(0.8, 1.25, batch)
    if filters == "mixed":
        t[r.random(batch) < 0.15] = 0.0                                          # some users want the most likely token
    k = np.where(on[:, 0], np.minimum(vocab, r.choice((1, 20, 40, 50, 100, 500), batch)), 0)
    p = np.where(on[:, 1], r.choice((0.5, 0.8, 0.9, 0.95, 0.99), batch), 1.0)
    m = np.where(on[:, 2], r.choice((0.02, 0.05, 0.1), batch), 0.0)
    s = {"case": case, "logits": logits, "uniform": torch.rand(batch, device=DEV, generator=g),
         "temperature": torch.from_numpy(t.astype(np.float32)).to(DEV), "top_k": torch.from_numpy(k.astype(np.int32)).to(DEV),
         "top_p": torch.from_numpy(p.astype(np.float32)).to(DEV), "min_p": torch.from_numpy(m.astype(np.float32)).to(DEV),
         "token": torch.empty(batch, dtype=torch.int32, device=DEV), "logprob": torch.empty(batch, device=DEV)}
    if own:
        from paper_2511_11729_amd import binding as hb
        s["workspace"] = torch.empty(hb.sample_workspace_bytes(batch, vocab), dtype=torch.uint8, device=DEV)
    return s


def _sample(s):
    if own:
        from paper_2511_11729_amd import binding as hb
        hb.sample(s["logits"], s["uniform"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                  logprob=s["logprob"], workspace=s["workspace"])
        return {"token": s["token"], "logprob": s["logprob"]}
    logits = s["logits"]
    batch, vocab = logits.shape
    value, order = logits.sort(dim=-1, descending=True, stable=True)                 # equal logits by index
    temperature = s["temperature"][:, None].double()
    greedy = temperature <= 0
    # 64 bits: sums over a vocabulary are compared with numbers that may lie next to them
    w = torch.exp((value.double() - value[:, :1].double()) / torch.where(greedy, torch.ones_like(temperature), temperature))
    rank = torch.arange(vocab, device=DEV)
    k = torch.where(s["top_k"] > 0, s["top_k"].clamp(max=vocab), vocab)[:, None]
    among = rank < k
    below = torch.cumsum(w, -1) - w
    p = s["top_p"][:, None].double()
    among &= (p >= 1) | (below < p * (w * among).sum(-1, keepdim=True)) | (rank == 0)
    among &= w >= s["min_p"][:, None].double()
    among &= ~greedy | (rank == 0)
    w = torch.empty_like(w).scatter_(-1, order, w * among)                       # by index again, without what is filtered out
    total = torch.cumsum(w, -1)
    token = (total <= s["uniform"][:, None].double() * total[:, -1:]).sum(-1, keepdim=True).clamp(max=vocab - 1)
    logprob = torch.log(w.gather(-1, token) / total[:, -1:])
    return {"token": token[:, 0].int(), "logprob": logprob[:, 0].float()}


def run(state):
    op = state["case"]["op"]
    return _attend(state) if op == "attend" else _evict(state) if op == "evict" else _sample(state)


# --------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "sample":
        return {"bytes": case["batch"] * (4.0 * case["vocab"] + 28), "flops": 3.0 * case["batch"] * case["vocab"]}
    lengths = _lengths(case, 1).astype(np.float64)
    n, row = float(lengths.sum()), case["d"] * _element(case)
    if case["op"] == "attend":
        # K, V and the records' weights in; weights and the newest records, q and out
        return {"bytes": n * case["n_kv"] * (2 * row + 8) + 8.0 * case["batch"] * case["n_q"] * case["d"], "flops": 4.0 * n * case["n_q"] * case["d"]}
    # records in; the rows and records that have to move, about the share of what lies behind the kept length that stays, in and out
    keep = _keep(case, lengths)
    share = np.where(keep < lengths, keep / lengths, 0.0)
    moved = float(((lengths - keep) * share).sum())
    heads = case["layers"] * case["n_kv"]
    return {"bytes": heads * (8 * n + moved * 2 * (2 * row + 8)), "flops": 0.0}


# --------------------------------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        return _exact_rows(s)
    return _exact_attention(s) if case["op"] == "attend" else _exact_eviction(s)


def _exact_attention(s):
    case = s["case"]
    n_kv, d, group = case["n_kv"], case["d"], case["n_q"] // case["n_kv"]
    out = torch.empty(case["batch"], case["n_q"], d, dtype=torch.float64, device=DEV)
    weight = s["track"][..., 0].view(torch.float32).double()
    position = s["track"][..., 1].clone()
    for b, n in enumerate(s["n"].tolist()):
        pages = s["table"][b, :-(-n // PAGE)].long()
        rows = s["view"][pages // s["ppb"], 0, :, pages % s["ppb"]].double()     # [page, K or V, KV head, slot, d]
        rows = rows.permute(1, 2, 0, 3, 4).reshape(2, n_kv, -1, d)[:, :, :n]
        logit = (rows[0][:, None] * s["q"][b].double().view(n_kv, group, 1, d)).sum(-1) / math.sqrt(d)
        p = torch.softmax(logit, -1)
        out[b] = (p[..., None] * rows[1][:, None]).sum(2).reshape(-1, d)
        w = weight[0, pages].transpose(0, 1).reshape(n_kv, -1).clone()
        w[:, n - 1] = 0
        w[:, :n] = w[:, :n] * case["decay"] + p.sum(1)
        weight[0, pages] = w.view(n_kv, -1, PAGE).transpose(0, 1)
        position[0, pages[-1], :, (n - 1) % PAGE] = s["position"][b]
    return {"out": out, "weight": weight, "position": position}


def _exact_eviction(s):
    case = s["case"]
    track, table = s["track"].cpu().numpy(), s["table"].cpu().numpy()
    if track[..., 0].size > 3e7:
        return None
    keep, count = s["keep"].tolist(), s["n"].tolist()
    moves = []
    for b in range(case["batch"]):
        n, k = count[b], min(count[b], keep[b])
        slot = np.arange(n)
        page, at = table[b, slot // PAGE], slot % PAGE
        for layer in range(case["layers"]):
            for c in range(case["n_kv"]):
                rec = track[layer, page, c, at]
                guarded = (rec[:, 1] < case["sink"]) | (rec[:, 1] >= n - case["recent"])
                best = np.lexsort((slot, -rec[:, 0].copy().view(np.float32).astype(np.float64), ~guarded))[:k]
                into, of = np.setdiff1d(slot[:k], best), np.sort(best[best >= k])
                track[layer, page[into], c, at[into]] = rec[of]
                moves.append(np.stack([np.full(len(into), layer), np.full(len(into), c), page[into], at[into], page[of], at[of]]))
    layer, c, p0, s0, p1, s1 = torch.from_numpy(np.concatenate(moves, 1)).to(DEV)
    cache = s["view"].clone()
    ppb = s["ppb"]
    cache[p0 // ppb, layer, :, p0 % ppb, c, s0] = s["view"][p1 // ppb, layer, :, p1 % ppb, c, s1]
    track = torch.from_numpy(track)
    return {"cache": cache, "weight": track[..., 0].contiguous().view(torch.float32), "position": track[..., 1],
            "n_left": torch.from_numpy(np.minimum(count, keep).astype(np.int32))}


def _exact_rows(s):
    logits = s["logits"].cpu().numpy().astype(np.float64)
    T, K, P, M, U = (s[x].cpu().numpy().astype(np.float64) for x in ("temperature", "top_k", "top_p", "min_p", "uniform"))
    token, logprob = np.zeros(len(logits), np.int32), np.zeros(len(logits))
    for i, row in enumerate(logits):
        if T[i] <= 0:
            token[i] = np.argmax(row)
            continue
        prob = np.exp((row - row.max()) / T[i])
        best = np.argsort(-row, kind="stable")
        if K[i] > 0:
            best = best[: int(K[i])]
        if P[i] < 1:
            before = np.concatenate(([0.0], np.cumsum(prob[best])))
            best = best[: max(1, np.searchsorted(before[:-1], P[i] * before[-1], side="left"))]
        best = np.sort(best[prob[best] >= M[i]])
        reach = np.cumsum(prob[best])
        token[i] = best[min(np.searchsorted(reach, U[i] * reach[-1], side="right"), len(best) - 1)]
        logprob[i] = math.log(prob[token[i]] / reach[-1])
    return {"token": token, "logprob": logprob}
