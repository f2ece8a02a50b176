"""The paged cache's operators as they are measured: their cases, inputs, plain forms in elementary torch operations,
their results in 64 bits, and the work a pass cannot do without.

  append   new tokens' keys and values into the pages of their sequences
  attend   attention of the new tokens over the paged cache
  weigh    the weight that the new tokens' attention gives to every cached token, added up per token
  evict    the tokens with the least weight leave the cache, those behind the budget take their slots

A case is a dict of plain values.  The sequences' lengths follow from it alone: the first holds len_hi tokens, the others
are spread over [len_lo, len_hi]; the first `long` sequences bring `new` tokens, the others `rest`.
"""
import math

import torch

own = False
DEV = "cuda:0"


def _case(kind, batch, h_q, h_kv, len_lo, len_hi, new=1, rest=None, long=1, d=128, page=64, causal=True, dtype="bf16", last=0,
          budget=0, sinks=0, recent=0):
    return dict(kind=kind, batch=batch, h_q=h_q, h_kv=h_kv, len_lo=len_lo, len_hi=len_hi, new=new, rest=new if rest is None else rest, long=long,
                d=d, page=page, causal=causal, dtype=dtype, last=last, budget=budget, sinks=sinks, recent=recent)


def listed():
    return [
        # one token of each sequence of a full serving batch
        dict(_case("append", 64, 32, 8, 1000, 8000), name="append_decode"),
        # the next pieces of four prompts, odd lengths, small pages
        dict(_case("append", 4, 32, 8, 2500, 9001, new=2047, page=16), name="append_chunk"),
        # one sequence at the start of its answer: latency
        dict(_case("attend", 1, 32, 8, 1000, 1000), name="decode_1k"),
        # a serving batch of unequal lengths, one token each: the cache is read once
        dict(_case("attend", 32, 32, 8, 4096, 32768), name="decode_32k"),
        # drafted tokens of eight sequences checked at once, group of 16, small pages
        dict(_case("attend", 8, 32, 2, 3000, 16000, new=5, page=16), name="draft_16k_g16"),
        # a piece of a long prompt against the cache before it
        dict(_case("attend", 1, 32, 8, 32768, 32768, new=2048), name="chunk_32k"),
        # a prompt's piece of odd length in one batch with seven decoding sequences
        dict(_case("attend", 8, 32, 8, 900, 11777, new=1501, rest=1), name="mixed_12k"),
        # fp32 tensors: two prompts' ends at head dimension 64, as in the fp32 parity configurations
        dict(_case("attend", 2, 4, 2, 700, 1024, new=333, d=64, dtype="fp32"), name="fp32_1k"),
        # the weights of a decoding batch's step
        dict(_case("weigh", 16, 32, 8, 2048, 16384), name="weigh_decode"),
        # the weights of a prompt's piece, head dimension 64
        dict(_case("weigh", 2, 16, 4, 6001, 16000, new=1999, d=64), name="weigh_chunk"),
        # a decoding batch whose caches have outgrown the budget by a few pages
        dict(_case("evict", 32, 32, 8, 4352, 4352, budget=4096, sinks=4, recent=256), name="evict_step"),
        # long prompts cut to a budget before their answers begin
        dict(_case("evict", 2, 32, 8, 20000, 32768, budget=4096, sinks=4, recent=512, page=16), name="evict_prompt"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "attend", "weigh", "weigh", "evict"])
    d, page = rng.choice([128, 128, 64]), rng.choice([16, 32, 64, 128])
    h_kv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 4, 4, 8, 16])
    while h_kv * g > 32:
        g //= 2
    h_q = h_kv * g
    if kind == "append":
        batch = _log_int(rng, 1, 128)
        new = _log_int(rng, 1, 8188 // batch) if rng.random() < 0.5 else 1
        lo = new + rng.randrange(0, 4000)
        return _case(kind, batch, h_q, h_kv, lo, lo + rng.randrange(0, 4000), new=new, long=batch, d=d, page=page,
                     dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if kind == "evict":
        batch = _log_int(rng, 1, 32)
        hi = _log_int(rng, 300, min(65536, 139264 // batch))
        budget = _log_int(rng, 64, hi)
        recent = rng.randrange(0, budget // 2)
        return _case(kind, batch, h_q, h_kv, (hi + budget) // 2, hi, d=d, page=page, budget=budget, sinks=rng.choice([0, 4]), recent=recent)
    if rng.random() < 0.15:
        hi = _log_int(rng, 40, 1500)
        new = _log_int(rng, 1, min(hi, 400))
        return _case(kind, rng.choice([1, 2, 3]), min(h_q, 4 * min(h_kv, 2)), min(h_kv, 2), max(new, hi // 2), hi, new=new, long=3, d=d, page=page,
                     causal=rng.random() < 0.7, dtype="fp32", last=rng.choice([0, 0, 16]))
    if rng.random() < 0.5:                                       # a few tokens a sequence, long caches
        batch = _log_int(rng, 1, 48)
        hi = _log_int(rng, 200, min(131072, 580000 // batch))
        return _case(kind, batch, h_q, h_kv, max(hi // 4, 40), hi, new=rng.choice([1, 1, 1, 2, 5]), long=batch, d=d, page=page)
    batch = rng.choice([1, 1, 2, 6])                             # a prompt's piece, alone or beside other sequences
    hi = _log_int(rng, 200, 32000 // batch)
    new = _log_int(rng, 20, min(hi, 2000))
    alone = rng.random() < 0.5
    return _case(kind, batch, h_q, h_kv, max(hi // 3, new if alone else 1), hi, new=new, rest=new if alone else 1, long=batch if alone else 1,
                 d=d, page=page, causal=rng.random() < 0.9, last=rng.choice([0, 0, 64]))


def _lengths(c):
    """Tokens in the cache and new tokens, for each sequence."""
    lens = [c["len_hi"] - int((c["len_hi"] - c["len_lo"]) * ((i * 0.6180339887) % 1.0)) for i in range(c["batch"])]
    return lens, [min(c["new"] if i < c["long"] else c["rest"], n) for i, n in enumerate(lens)]


def _elem(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    lens, news = _lengths(c)
    P, h_kv, d, el = c["page"], c["h_kv"], c["d"], _elem(c)
    per = [-(-n // P) for n in lens]
    n_pages, width = sum(per) + 3, max(per)
    ids = torch.randperm(n_pages, generator=gen, device=DEV)[: sum(per)].tolist()
    table, at = [], 0
    for k in per:                                                # -1: no page
        table.append(ids[at: at + k] + [-1] * (width - k))
        at += k
    starts = [0]
    for m in news:
        starts.append(starts[-1] + m)
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    rand = lambda *sh: torch.randn(sh, generator=gen, device=DEV, dtype=torch.float32)  # noqa: E731
    s = dict(c=c, rows=starts[-1], T=max(news), L=max(lens), table=whole(table), lens=whole(lens), row_start=whole(starts))
    s["k"] = rand(n_pages, h_kv, P, d).to(el)
    s["v"] = rand(n_pages, h_kv, P, d).to(el)
    if c["kind"] == "append":
        s["k_new"], s["v_new"] = rand(s["rows"], h_kv, d).to(el), rand(s["rows"], h_kv, d).to(el)
        s["seen"] = s["lens"] + 100                              # a hundred tokens were evicted before
        s["weights"], s["pos"] = rand(n_pages, h_kv, P).exp(), torch.zeros((n_pages, h_kv, P), dtype=torch.int32, device=DEV)
    if c["kind"] in ("attend", "weigh"):
        # logits of standard deviation 2
        s["q"] = (2.0 * rand(s["rows"], c["h_q"], d)).to(el)
    if c["kind"] == "weigh":
        s["weights"] = rand(n_pages, h_kv, P).exp() * (s["rows"] / sum(lens))   # about what one pass adds
        s["lse"] = _unpad(s, _scores(s).logsumexp(-1).view(c["batch"], h_kv, s["T"], -1).transpose(1, 2).flatten(2)).contiguous()
    if c["kind"] == "evict":
        s["seen"] = s["lens"] + 1000
        # weights over several orders of magnitude, a tenth of them zero; positions in no order, as earlier evictions leave them
        w = (2.0 * rand(n_pages, h_kv, P)).exp()
        s["weights"] = torch.where(torch.rand(w.shape, generator=gen, device=DEV) < 0.1, torch.zeros_like(w), w)
        s["pos"] = torch.zeros((n_pages, h_kv, P), dtype=torch.int32, device=DEV)
        for b, n in enumerate(lens):
            old = torch.rand((h_kv, n + 1000), generator=gen, device=DEV).argsort(-1)[:, :n].to(torch.int32)
            at = torch.arange(n, device=DEV)
            s["pos"][s["table"][b, at // P].long()[None], torch.arange(h_kv, device=DEV)[:, None], (at % P)[None]] = old
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _flat(s):
    """[batch, h_kv, L]: the row that a slot's token has among all (page, head, token) rows."""
    c = s["c"]
    at = torch.arange(s["L"], device=DEV)
    page = s["table"].long().clamp(min=0)[:, at // c["page"]]
    head = torch.arange(c["h_kv"], device=DEV)
    return (page[:, None, :] * c["h_kv"] + head[None, :, None]) * c["page"] + (at % c["page"])


def _scores(s):
    """[batch, h_kv, T * g, L]: logits, -inf where a token is not visible."""
    c = s["c"]
    B, h_kv, T, L, d = c["batch"], c["h_kv"], s["T"], s["L"], c["d"]
    t = torch.arange(T, device=DEV)
    start, n = s["row_start"].long(), s["lens"].long()
    q = s["q"][(start[:-1, None] + t).clamp(max=s["rows"] - 1)].float()                         # [B, T, h_q, d]
    q = q.view(B, T, h_kv, -1, d).transpose(1, 2).reshape(B, h_kv, -1, d)
    x = torch.matmul(q, s["k"].view(-1, d)[_flat(s)].float().transpose(-1, -2)) * (1.0 / math.sqrt(d))
    end = n[:, None] - (start[1:] - start[:-1])[:, None] + t if c["causal"] else (n[:, None] - 1).expand(B, T)
    seen = torch.arange(L, device=DEV) <= torch.minimum(end, n[:, None] - 1)[..., None]          # [B, T, L]
    seen = seen[:, None, :, None].expand(B, 1, T, c["h_q"] // h_kv, L).reshape(B, 1, -1, L)
    return x.masked_fill_(~seen, -math.inf)


def _unpad(s, x):
    """The packed rows of x [batch, T, ...]."""
    r = torch.arange(s["rows"], device=DEV)
    start = s["row_start"].long()
    b = torch.searchsorted(start[1:].contiguous(), r, right=True)
    return x[b, r - start[b]]


def _attend(s):
    c = s["c"]
    B, h_kv, T, d = c["batch"], c["h_kv"], s["T"], c["d"]
    x = _scores(s)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = s["v"].view(-1, d)[_flat(s)].float()
    v = torch.where((torch.arange(s["L"], device=DEV) < s["lens"][:, None])[:, None, :, None], v, torch.zeros((), device=DEV))
    o = torch.matmul(x, v) / total
    rows = lambda y: _unpad(s, y.view(B, h_kv, T, c["h_q"] // h_kv, -1).transpose(1, 2).flatten(2, 3))  # noqa: E731
    return {"o": rows(o).to(s["q"].dtype), "lse": rows(top + total.log())[..., 0]}


def _weigh(s):
    c = s["c"]
    B, h_kv, T, L = c["batch"], c["h_kv"], s["T"], s["L"]
    t = torch.arange(T, device=DEV)
    start = s["row_start"].long()
    new = (start[1:] - start[:-1])[:, None]
    first = new - c["last"] if c["last"] else torch.zeros_like(new)
    lse = s["lse"][(start[:-1, None] + t).clamp(max=s["rows"] - 1)]                              # [B, T, h_q]
    lse = lse.masked_fill(((t >= new) | (t < first))[..., None], math.inf)                       # rows that do not weigh
    p = _scores(s).sub_(lse.view(B, T, h_kv, -1).transpose(1, 2).reshape(B, h_kv, -1, 1)).exp_().sum(-2)
    inside = (torch.arange(L, device=DEV) < s["lens"][:, None])[:, None].expand(B, h_kv, L)
    w = s["weights"].clone()
    w.view(-1).index_add_(0, _flat(s).reshape(-1), torch.where(inside, p, torch.zeros((), device=DEV)).reshape(-1))
    return {"weights": w}


def _evict(s):
    c = s["c"]
    B, h_kv, L, d, budget = c["batch"], c["h_kv"], s["L"], c["d"], c["budget"]
    w, pos, lens = s["weights"].clone(), s["pos"].clone(), s["lens"].clone()
    flat, n = _flat(s), lens.long()[:, None, None]
    at = torch.arange(L, device=DEV).expand(B, h_kv, L)
    p, x = pos.view(-1)[flat], w.view(-1)[flat]
    x = torch.where(torch.isnan(x), torch.full_like(x, -1.0), x)
    x = torch.where((p < c["sinks"]) | (p >= s["seen"][:, None, None] - c["recent"]), torch.full_like(x, math.inf), x)
    x = torch.where(at < n, x, torch.full_like(x, -math.inf))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    left = torch.minimum(n, torch.full_like(n, budget))
    kept = torch.zeros_like(x, dtype=torch.bool).scatter_(-1, order, at < left)
    # the j-th free slot before the budget takes the j-th kept token behind it
    hole, mover = ~kept & (at < left), kept & (at >= left)
    holes = torch.sort((~hole).to(torch.int8), dim=-1, stable=True).indices
    movers = torch.sort((~mover).to(torch.int8), dim=-1, stable=True).indices
    moved = at < hole.sum(-1, keepdim=True)
    src = at.clone().scatter_(-1, holes, torch.where(moved, movers, holes))[..., :budget]
    live = at[..., :src.shape[-1]] < left
    # slots behind a sequence's end have no row of their own: the rows of live slots only
    to = torch.where(live, flat[..., :src.shape[-1]], flat[..., :1])
    frm = torch.where(live, flat.gather(-1, src), flat.gather(-1, src[..., :1]))
    for x in (s["k"].view(-1, d), s["v"].view(-1, d), w.view(-1), pos.view(-1)):
        x[to.reshape(-1)] = x[frm.reshape(-1)]
    out = torch.full((B, h_kv, budget), -1, dtype=torch.int32, device=DEV)
    out[..., :src.shape[-1]] = torch.where(live, src, torch.full_like(src, -1)).to(torch.int32)
    return {"k": s["k"], "v": s["v"], "weights": w, "pos": pos, "lens": left[:, 0, 0].to(torch.int32), "src": out}


def _append(s):
    c = s["c"]
    P, h_kv, d = c["page"], c["h_kv"], c["d"]
    r = torch.arange(s["rows"], device=DEV)
    start = s["row_start"].long()
    b = torch.searchsorted(start[1:].contiguous(), r, right=True)
    back = start[1:][b] - r                                      # 1: the sequence's newest token
    slot = s["lens"].long()[b] - back
    page = s["table"].long()[b, slot // P]
    to = ((page[:, None] * h_kv + torch.arange(h_kv, device=DEV)) * P + (slot % P)[:, None]).reshape(-1)
    s["k"].view(-1, d)[to] = s["k_new"].reshape(-1, d)
    s["v"].view(-1, d)[to] = s["v_new"].reshape(-1, d)
    s["weights"].view(-1)[to] = 0.0
    s["pos"].view(-1)[to] = (s["seen"].long()[b] - back).to(torch.int32)[:, None].expand(-1, h_kv).reshape(-1)
    return {"k": s["k"], "v": s["v"], "weights": s["weights"], "pos": s["pos"]}


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _own(s):
    from paper_2605_18753_amd import binding as B
    c = s["c"]
    if "p" not in s:                                             # what a program keeps: the parameters, the scratch, the outputs' buffers
        s["cache"] = B.PagedCache(s["k"], s["v"], s["table"], s["lens"])
        s["p"] = B.make_paged_params(s["cache"], s["rows"], c["h_q"], causal=c["causal"])
        s["ws"] = B.alloc_paged_workspace(s["p"], DEV, evict=c["kind"] == "evict")
        if c["kind"] == "attend":
            s["o"] = torch.empty_like(s["q"])
            s["lse_out"] = torch.empty((s["rows"], c["h_q"]), dtype=torch.float32, device=DEV)
        if c["kind"] == "evict":
            s["src"] = torch.empty((c["batch"], c["h_kv"], c["budget"]), dtype=torch.int32, device=DEV)
    p, cache = s["p"], s["cache"]
    if c["kind"] == "attend":
        B.dash_paged_attend(p, cache, s["q"], s["row_start"], s["o"], s["ws"], lse=s["lse_out"])
        return {"o": s["o"], "lse": s["lse_out"]}
    if c["kind"] == "weigh":
        cache.weights = s["weights"].clone()
        B.dash_paged_weigh(p, cache, s["q"], s["row_start"], s["lse"], s["ws"], last=c["last"])
        return {"weights": cache.weights}
    if c["kind"] == "evict":
        cache.weights, cache.pos, cache.lens, cache.seen = s["weights"].clone(), s["pos"].clone(), s["lens"].clone(), s["seen"]
        B.dash_paged_evict(p, cache, c["budget"], s["ws"], sinks=c["sinks"], recent=c["recent"], src=s["src"])
        return {"k": cache.k, "v": cache.v, "weights": cache.weights, "pos": cache.pos, "lens": cache.lens, "src": s["src"]}
    cache.weights, cache.pos, cache.seen = s["weights"], s["pos"], s["seen"]
    B.dash_paged_append(p, cache, s["k_new"], s["v_new"], s["row_start"])
    return {"k": cache.k, "v": cache.v, "weights": cache.weights, "pos": cache.pos}


def run(state):
    if own:
        return _own(state)
    return {"append": _append, "attend": _attend, "weigh": _weigh, "evict": _evict}[state["c"]["kind"]](state)


# ---- work ------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    lens, news = _lengths(c)
    es = 2 if c["dtype"] == "bf16" else 4
    row = c["h_kv"] * c["d"] * es                                # a token's keys, or values
    q_row = c["h_q"] * c["d"] * es
    if c["kind"] == "append":
        return {"bytes": sum(news) * (4.0 * row + 8.0 * c["h_kv"]), "flops": 0}
    if c["kind"] == "evict":
        moves = sum(min(n, c["budget"]) * max(n - c["budget"], 0) / n for n in lens)   # kept tokens are spread evenly over the slots
        return {"bytes": c["h_kv"] * (8.0 * sum(lens) + 4.0 * c["batch"] * c["budget"]) + moves * (4.0 * row + 16.0 * c["h_kv"]), "flops": 0}
    pairs = keys = rows = 0.0
    for n, m in zip(lens, news):
        if c["kind"] == "weigh" and c["last"]:
            m = min(m, c["last"])
        rows += m
        pairs += m * n - (m * (m - 1) / 2 if c["causal"] else 0)
        keys += n
    if c["kind"] == "weigh":
        return {"bytes": keys * (row + 8.0 * c["h_kv"]) + rows * (q_row + 4.0 * c["h_q"]), "flops": 2.0 * pairs * c["h_q"] * c["d"]}
    return {"bytes": 2.0 * keys * row + rows * (2.0 * q_row + 4.0 * c["h_q"]), "flops": 4.0 * pairs * c["h_q"] * c["d"]}


# ---- the definitions in 64 bits, one sequence and one kv-head after the other ----------------------------------------
def exact(case, seed):
    c = case
    s = prepare(c, seed)
    lens, news = _lengths(c)
    P, g, d = c["page"], c["h_q"] // c["h_kv"], c["d"]
    q0 = 0
    out = {}
    if c["kind"] == "attend":
        out = {"o": torch.zeros((s["rows"], c["h_q"], d), dtype=torch.float64, device=DEV),
               "lse": torch.zeros((s["rows"], c["h_q"]), dtype=torch.float64, device=DEV)}
    elif c["kind"] == "weigh":
        out = {"weights": s["weights"].double()}
    elif c["kind"] == "evict":
        out = {"k": s["k"], "v": s["v"], "weights": s["weights"].clone(), "pos": None, "lens": None, "src": None}
    else:
        out = {"k": s["k"], "v": s["v"], "weights": s["weights"].clone(), "pos": None}
    for b, (n, m) in enumerate(zip(lens, news)):
        at = torch.arange(n, device=DEV)
        page, off = s["table"][b].long()[at // P], at % P
        for h in range(c["h_kv"]):
            if c["kind"] == "append":
                for name in ("k", "v"):
                    out[name][page[n - m:], h, off[n - m:]] = s[name + "_new"][q0:q0 + m, h]
                out["weights"][page[n - m:], h, off[n - m:]] = 0
                continue
            if c["kind"] == "evict":
                if n <= c["budget"]:
                    continue
                w, pos = s["weights"][page, h, off].double().cpu(), s["pos"][page, h, off].cpu()
                safe = (pos < c["sinks"]) | (pos >= n + 1000 - c["recent"])
                ranks = sorted(range(n), key=list(zip((~safe).tolist(), (-w).tolist(), range(n))).__getitem__)
                kept = sorted(ranks[: c["budget"]])
                among = set(kept)
                into = [i for i in range(c["budget"]) if i not in among]
                come = [i for i in kept if i >= c["budget"]]
                i, j = torch.tensor(into, device=DEV, dtype=torch.long), torch.tensor(come, device=DEV, dtype=torch.long)
                for name in ("k", "v", "weights"):
                    out[name][page[i], h, off[i]] = out[name][page[j], h, off[j]]
                continue
            K = s["k"][page, h, off].double()
            Q = s["q"][q0:q0 + m, h * g:(h + 1) * g].double().permute(1, 0, 2).reshape(g * m, d)
            x = torch.matmul(Q, K.t().contiguous()).view(g, m, n) / math.sqrt(d)
            if c["causal"]:
                late = torch.ones((m, n), dtype=torch.bool, device=DEV).triu(n - m + 1)
                x.masked_fill_(late, -math.inf)
            if c["kind"] == "attend":
                l = torch.logsumexp(x, -1)
                x = torch.exp(x - l[..., None]).view(g * m, n)
                out["o"][q0:q0 + m, h * g:(h + 1) * g] = torch.matmul(x, s["v"][page, h, off].double()).view(g, m, d).permute(1, 0, 2)
                out["lse"][q0:q0 + m, h * g:(h + 1) * g] = l.t()
            else:
                x = torch.exp(x - s["lse"][q0:q0 + m, h * g:(h + 1) * g].double().t()[..., None])
                if c["last"]:
                    x = x[:, -min(c["last"], m):]
                out["weights"][page, h, off] += x.sum((0, 1))
            del x
        q0 += m
    return out
