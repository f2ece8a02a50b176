"""Rotary positions and the paged cache in 4 bits as they are measured: cases, inputs, plain forms in elementary torch operations,
results in 64 bits, and the work a pass cannot do without.

  rotary       queries and keys turned by their tokens' positions, or gradients turned back
  append_rot   new tokens into a paged cache, their keys (and the step's queries) turned on the way
  append4      the same into a cache that holds 4 bits a number, which is then read back as bf16 or fp32 pages
  attend4      attention of the new tokens over the cache in 4 bits

Rotary positions: pair i of the first `rot` elements of a head turns by position * theta_i, theta_i = base^(-2i / rot) (scaled for long contexts:
`_thetas`), its numbers multiplied by `mscale`.
4 bits: 32 numbers of a row share a power of two, 2^e; each is held as one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign, nearest first, ties to the even
code.  e is floor(log2 of the largest) - 2, one more where the largest would be above 7.25 (it is held as 6), within -120 .. 125.

A case is a dict of plain values.  The sequences' lengths follow from it alone: the first holds len_hi tokens, the others
are spread over [len_lo, len_hi]; the first `long` sequences bring `new` tokens, the others `rest`.
"""
import math

import torch

own = False
DEV = "cuda:0"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(kind, batch, h_q, h_kv, len_lo, len_hi, new=1, rest=None, long=1, d=128, page=64, causal=True, dtype="bf16",
          rot=0, layout="halves", base=10000.0, scaling="", factor=1.0, mscale=1.0, far=0, inverse=False):
    return dict(kind=kind, batch=batch, h_q=h_q, h_kv=h_kv, len_lo=len_lo, len_hi=len_hi, new=new, rest=new if rest is None else rest, long=long,
                d=d, page=page, causal=causal, dtype=dtype, rot=rot, layout=layout, base=base, scaling=scaling, factor=factor, mscale=mscale,
                far=far, inverse=inverse)


def listed():
    return [
        # queries and keys of a training batch
        dict(_case("rotary", 4, 16, 16, 8192, 8192, rot=128), name="rotary_train_8k"),
        # gradients turned back: fp32, half of each head, neighbours as pairs, frequencies scaled by parts, positions far along, odd length
        dict(_case("rotary", 2, 16, 4, 3001, 3001, d=64, dtype="fp32", rot=32, layout="adjacent", scaling="parts", factor=8.0, mscale=1.2, far=500000,
                   inverse=True), name="rotary_grad_3k"),
        # one token of each sequence of a full serving batch
        dict(_case("append_rot", 64, 32, 8, 1000, 8000, rot=128), name="append_rot_decode"),
        # the next pieces of four long prompts, odd lengths, small pages, half of each head
        dict(_case("append_rot", 4, 32, 8, 2500, 9001, new=2047, page=16, rot=64, layout="adjacent", scaling="linear", factor=4.0, far=100000),
             name="append_rot_chunk"),
        # first tokens of the answers of a serving batch, short caches
        dict(_case("append4", 64, 32, 8, 1, 120, rot=128, base=500000.0), name="append4_decode"),
        # pieces of four prompts, odd lengths, small pages
        dict(_case("append4", 4, 32, 8, 2047, 2500, new=2047, page=16, rot=128, scaling="base", factor=4.0), name="append4_chunk"),
        # one sequence at the start of its answer: latency
        dict(_case("attend4", 1, 32, 8, 1000, 1000), name="attend4_decode_1k"),
        # a serving batch of unequal lengths, one token each: the cache is read once
        dict(_case("attend4", 32, 32, 8, 4096, 32768), name="attend4_decode_32k"),
        # drafted tokens of eight sequences checked at once, group of 16, small pages
        dict(_case("attend4", 8, 32, 2, 3000, 16000, new=5, page=16), name="attend4_draft_16k_g16"),
        # a piece of a long prompt against the cache before it
        dict(_case("attend4", 1, 32, 8, 32768, 32768, new=2048), name="attend4_chunk_32k"),
        # a prompt's piece of odd length in one batch with seven decoding sequences, head dimension 64
        dict(_case("attend4", 8, 32, 8, 900, 11777, new=1501, rest=1, d=64), name="attend4_mixed_12k_d64"),
        # fp32 queries: two prompts' ends at head dimension 64, as in the fp32 parity configurations
        dict(_case("attend4", 2, 4, 2, 700, 1024, new=333, d=64, dtype="fp32"), name="attend4_fp32_1k"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "append_rot", "append_rot", "append4", "append4", "attend4", "attend4", "attend4", "attend4", "attend4"])
    d, page = rng.choice([128, 128, 64]), rng.choice([16, 32, 64, 128])
    h_kv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 4, 4, 8, 16])
    while h_kv * g > 32:
        g //= 2
    h_q = h_kv * g
    turn = {}
    if kind != "attend4":
        scaling = rng.choice(["", "", "linear", "base", "parts"])
        turn = dict(rot=rng.choice([d, d, d, 16 * rng.randint(1, d // 16)]), layout=rng.choice(["halves", "halves", "adjacent"]), base=rng.choice([1e4, 5e5]),
                    scaling=scaling, factor=rng.choice([2.0, 4.0, 32.0]) if scaling else 1.0, mscale=rng.choice([1.0, 1.0, 1.25]),
                    far=rng.choice([0, 0, rng.randrange(1000, 1000000)]))
    if kind == "rotary":
        batch = _log_int(rng, 1, 64)
        n = _log_int(rng, 1, 131072 // batch)
        while batch * n * (h_q + h_kv) * d > 4 * 32 * 8192 * 128:
            n = (n + 1) // 2
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        if dtype == "fp32":
            n = (n + 1) // 2
        return _case(kind, batch, h_q, h_kv, n, n, d=d, dtype=dtype, inverse=rng.random() < 0.5, **turn)
    if kind == "append_rot":
        batch = _log_int(rng, 1, 128)
        new = _log_int(rng, 1, 8188 // batch) if rng.random() < 0.5 else 1
        lo = new + rng.randrange(0, 2000)
        return _case(kind, batch, h_q, h_kv, lo, lo + rng.randrange(0, 2000), new=new, long=batch, d=d, page=page, dtype=rng.choice(["bf16", "bf16", "fp32"]), **turn)
    if kind == "append4":
        batch = _log_int(rng, 1, 64)
        new = _log_int(rng, 1, 8188 // batch) if rng.random() < 0.5 else 1
        lo = new + rng.randrange(0, 60)
        return _case(kind, batch, h_q, h_kv, lo, lo + rng.randrange(0, 60), new=new, long=batch, d=d, page=page, dtype=rng.choice(["bf16", "bf16", "fp32"]), **turn)
    if rng.random() < 0.15:
        hi = _log_int(rng, 40, 1500)
        new = _log_int(rng, 1, min(hi, 400))
        return _case(kind, rng.choice([1, 2, 3]), min(h_q, 4 * min(h_kv, 2)), min(h_kv, 2), max(new, hi // 2), hi, new=new, long=3, d=d, page=page,
                     causal=rng.random() < 0.7, dtype="fp32")
    if rng.random() < 0.5:                                       # a few tokens a sequence, long caches
        batch = _log_int(rng, 1, 48)
        hi = _log_int(rng, 200, min(131072, 580000 // batch))
        return _case(kind, batch, h_q, h_kv, max(hi // 4, 40), hi, new=rng.choice([1, 1, 1, 2, 5]), long=batch, d=d, page=page)
    batch = rng.choice([1, 1, 2, 6])                             # a prompt's piece, alone or beside other sequences
    hi = _log_int(rng, 200, 32000 // batch)
    new = _log_int(rng, 20, min(hi, 2000))
    alone = rng.random() < 0.5
    return _case(kind, batch, h_q, h_kv, max(hi // 3, new if alone else 1), hi, new=new, rest=new if alone else 1, long=batch if alone else 1,
                 d=d, page=page, causal=rng.random() < 0.9)


def _lengths(c):
    """Tokens in the cache and new tokens, for each sequence."""
    lens = [c["len_hi"] - int((c["len_hi"] - c["len_lo"]) * ((i * 0.6180339887) % 1.0)) for i in range(c["batch"])]
    return lens, [min(c["new"] if i < c["long"] else c["rest"], n) for i, n in enumerate(lens)]


def _elem(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


ORIGINAL, LOW, HIGH = 8192.0, 1.0, 4.0                           # of scaling by parts: the context trained on, turns over it between which the ramp lies


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    h_q, h_kv, d, el = c["h_q"], c["h_kv"], c["d"], _elem(c)
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    rand = lambda *sh: torch.randn(sh, generator=gen, device=DEV, dtype=torch.float32)  # noqa: E731
    # keys of trained models have a few dimensions much larger than the others
    loud = (0.7 * rand(h_kv, 1, d)).exp()
    if c["kind"] == "rotary":
        n = c["len_hi"]
        s = dict(c=c, q=rand(c["batch"], h_q, n, d).to(el), k=(rand(c["batch"], h_kv, n, d) * loud).to(el))
        if c["far"]:                                             # positions of each sequence's own start, in order
            s["pos"] = (torch.randint(0, c["far"], (c["batch"], 1), generator=gen, device=DEV) + torch.arange(n, device=DEV)).to(torch.int32)
        return s
    lens, news = _lengths(c)
    P = c["page"]
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
    s = dict(c=c, rows=starts[-1], T=max(news), L=max(lens), table=whole(table), lens=whole(lens), row_start=whole(starts))
    rows = s["rows"]
    if c["kind"] == "append_rot":
        s["k"], s["v"] = rand(n_pages, h_kv, P, d).to(el), rand(n_pages, h_kv, P, d).to(el)
        s["weights"], s["pos"] = rand(n_pages, h_kv, P).exp(), torch.zeros((n_pages, h_kv, P), dtype=torch.int32, device=DEV)
    else:
        for name, f in (("k", loud), ("v", None)):
            codes = torch.empty((n_pages, h_kv, P, d // 2), dtype=torch.uint8, device=DEV)
            scales = torch.empty((n_pages, h_kv, P, d // 32), dtype=torch.uint8, device=DEV)
            step = max(1, (1 << 26) // (h_kv * P * d))
            for i in range(0, n_pages, step):                    # a part of the pool at a time
                x = rand(min(step, n_pages - i), h_kv, P, d)
                codes[i:i + step], scales[i:i + step] = _quantise(x if f is None else x * f)
            s[name + "_codes"], s[name + "_scales"] = codes, scales
    if c["kind"] == "attend4":
        s["q"] = (2.0 * rand(rows, h_q, d) / loud.mean()).to(el)
        return s
    s["q"] = rand(rows, h_q, d).to(el)
    s["k_new"], s["v_new"] = (rand(rows, h_kv, d) * loud.transpose(0, 1)).to(el), rand(rows, h_kv, d).to(el)
    s["seen"] = s["lens"] + (torch.randint(0, c["far"], (c["batch"],), generator=gen, device=DEV).to(torch.int32) if c["far"] else 0)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _thetas(c):
    """Radians a token, one for each pair, in 64 bits."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    base = c["base"] * c["factor"] ** (c["rot"] / (c["rot"] - 2)) if c["scaling"] == "base" else c["base"]
    theta = base ** (-2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        theta = theta / c["factor"]
    if c["scaling"] == "parts":                                  # fast pairs stay, slow ones are divided by the factor
        keep = ((ORIGINAL * theta / (2.0 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        theta = theta * ((1.0 - keep) / c["factor"] + keep)
    return theta


def _turn(c, x, pos, f=torch.float32):
    """x [..., d] turned at positions pos, which has x's leading sizes or broadcasts to them, in type f."""
    rot, half = c["rot"], c["rot"] // 2
    a = pos[..., None].double() * _thetas(c)
    cos, sin = (a.cos() * c["mscale"]).to(f), (a.sin() * (-c["mscale"] if c["inverse"] else c["mscale"])).to(f)
    y = x.to(f, copy=True)
    one, two = (y[..., :half], y[..., half:rot]) if c["layout"] == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2])
    one_new, two_new = one * cos - two * sin, two * cos + one * sin
    one.copy_(one_new)
    two.copy_(two_new)
    return y


def _quantise(x):
    """Codes (the even element low) and scales (e + 127), both uint8, of x [..., d]."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    e = torch.frexp(top)[1] - 3
    e = (e + (torch.ldexp(top, -e) > 7.25)).clamp(-120, 125)
    e = torch.where(top > 0, e, torch.full_like(e, -120))
    t = torch.ldexp(b, -e[..., None])
    code = torch.signbit(t).to(torch.uint8) * 8
    t = t.abs()
    for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (t >= border) if up else (t > border)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What they stand for, fp32 [..., d]."""
    half = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float32, device=codes.device)
    pair = torch.stack((half.repeat(16), half.repeat_interleave(16)), -1)                        # of a byte
    x = pair.index_select(0, codes.reshape(-1).int()).view(*codes.shape[:-1], -1, 32)
    return torch.ldexp(x, (scales.int() - 127)[..., None]).flatten(-2)


def _flat(s):
    """[batch, h_kv, L]: the row that a slot's token has among all (page, head, token) rows."""
    c = s["c"]
    at = torch.arange(s["L"], device=DEV)
    page = s["table"].long().clamp(min=0)[:, at // c["page"]]
    head = torch.arange(c["h_kv"], device=DEV)
    return (page[:, None, :] * c["h_kv"] + head[None, :, None]) * c["page"] + (at % c["page"])


def _unpad(s, x):
    """The packed rows of x [batch, T, ...]."""
    r = torch.arange(s["rows"], device=DEV)
    start = s["row_start"].long()
    b = torch.searchsorted(start[1:].contiguous(), r, right=True)
    return x[b, r - start[b]]


def _attend4(s):
    c = s["c"]
    B, h_kv, T, L, d = c["batch"], c["h_kv"], s["T"], s["L"], c["d"]
    flat = _flat(s)
    cached = lambda name: _values(s[name + "_codes"].view(-1, d // 2)[flat], s[name + "_scales"].view(-1, d // 32)[flat])  # noqa: E731
    t = torch.arange(T, device=DEV)
    start, n = s["row_start"].long(), s["lens"].long()
    q = s["q"][(start[:-1, None] + t).clamp(max=s["rows"] - 1)].float()                         # [B, T, h_q, d]
    q = q.view(B, T, h_kv, -1, d).transpose(1, 2).reshape(B, h_kv, -1, d)
    x = torch.matmul(q, cached("k").transpose(-1, -2)) * (1.0 / math.sqrt(d))
    end = n[:, None] - (start[1:] - start[:-1])[:, None] + t if c["causal"] else (n[:, None] - 1).expand(B, T)
    seen = torch.arange(L, device=DEV) <= torch.minimum(end, n[:, None] - 1)[..., None]          # [B, T, L]
    x.masked_fill_(~seen[:, None, :, None].expand(B, 1, T, c["h_q"] // h_kv, L).reshape(B, 1, -1, L), -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    v = cached("v")
    v = torch.where((torch.arange(L, device=DEV) < s["lens"][:, None])[:, None, :, None], v, torch.zeros((), device=DEV))
    o = torch.matmul(x, v) / total
    rows = lambda y: _unpad(s, y.view(B, h_kv, T, c["h_q"] // h_kv, -1).transpose(1, 2).flatten(2, 3))  # noqa: E731
    return {"o": rows(o).to(s["q"].dtype), "lse": rows(top + total.log())[..., 0]}


def _places(s):
    """The rows that the new tokens' keys have among all (page, head, token) rows [rows, h_kv], and their positions."""
    c = s["c"]
    r = torch.arange(s["rows"], device=DEV)
    start = s["row_start"].long()
    b = torch.searchsorted(start[1:].contiguous(), r, right=True)
    back = start[1:][b] - r                                      # 1: the sequence's newest token
    slot = s["lens"].long()[b] - back
    page = s["table"].long()[b, slot // c["page"]]
    to = (page[:, None] * c["h_kv"] + torch.arange(c["h_kv"], device=DEV)) * c["page"] + (slot % c["page"])[:, None]
    return to, s["seen"].long()[b] - back


def _append_rot(s):
    c = s["c"]
    d, el = c["d"], _elem(c)
    to, pos = _places(s)
    s["k"].view(-1, d)[to] = _turn(c, s["k_new"], pos[:, None]).to(el)
    s["v"].view(-1, d)[to] = s["v_new"]
    s["weights"].view(-1)[to] = 0.0
    s["pos"].view(-1)[to] = pos.to(torch.int32)[:, None].expand(-1, c["h_kv"])
    return {"q": _turn(c, s["q"], pos[:, None]).to(el), "k": s["k"], "v": s["v"], "weights": s["weights"], "pos": s["pos"]}


def _append4(s):
    c = s["c"]
    d, el = c["d"], _elem(c)
    to, pos = _places(s)
    # turned in 64 bits: a number next to the border between two codes must fall on the right side
    for name, x in (("k", _turn(c, s["k_new"], pos[:, None], torch.float64)), ("v", s["v_new"].float())):
        codes, scales = _quantise(x)
        s[name + "_codes"].view(-1, d // 2)[to] = codes
        s[name + "_scales"].view(-1, d // 32)[to] = scales
    pages = {name: _values(s[name + "_codes"], s[name + "_scales"]).to(el) for name in ("k", "v")}
    return {"q": _turn(c, s["q"], pos[:, None]).to(el), **pages}


def _rotary(s):
    c = s["c"]
    pos = s["pos"][:, None] if "pos" in s else torch.arange(c["len_hi"], device=DEV)
    return {"q": _turn(c, s["q"], pos).to(_elem(c)), "k": _turn(c, s["k"], pos).to(_elem(c))}


# ---- the framework's calls -------------------------------------------------------------------------------------------
def _own(s):
    from paper_2605_18753_amd import binding as B
    c = s["c"]
    if "ready" not in s:                                         # what a program keeps: plans, parameters, scratch, the outputs' buffers
        s["ready"] = True
        if c["kind"] != "attend4":
            s["rotary"] = B.make_rotary(c["rot"], DEV, layout=c["layout"], base=c["base"], scaling=c["scaling"] or None, factor=c["factor"],
                                        original=ORIGINAL, low=LOW, high=HIGH, mscale=c["mscale"])
            s["q_out"] = torch.empty_like(s["q"])
        if c["kind"] == "rotary":
            s["k_out"] = torch.empty_like(s["k"])
        elif c["kind"] == "append_rot":
            s["cache"] = B.PagedCache(s["k"], s["v"], s["table"], s["lens"], s["weights"], s["pos"], s["seen"])
            s["p"] = B.make_paged_params(s["cache"], s["rows"], c["h_q"])
        else:
            s["cache"] = B.PagedCache4(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], s["table"], s["lens"], seen=s.get("seen"))
            s["p"] = B.make_paged4_params(s["cache"], s["rows"], c["h_q"], dtype=_elem(c), causal=c["causal"])
        if c["kind"] == "append4":
            s["k"], s["v"] = (torch.empty((*s["k_codes"].shape[:3], c["d"]), dtype=_elem(c), device=DEV) for _ in range(2))
        if c["kind"] == "attend4":
            s["ws"] = B.alloc_paged4_workspace(s["p"], DEV)
            s["o"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty((s["rows"], c["h_q"]), dtype=torch.float32, device=DEV)
    if c["kind"] == "rotary":
        B.dash_rotary(s["rotary"], s["q"], s["q_out"], s["k"], s["k_out"], pos=s.get("pos"), inverse=c["inverse"])
        return {"q": s["q_out"], "k": s["k_out"]}
    p, cache = s["p"], s["cache"]
    if c["kind"] == "append_rot":
        B.dash_paged_append_rotary(p, cache, s["rotary"], s["k_new"], s["v_new"], s["row_start"], q=s["q"], q_out=s["q_out"])
        return {"q": s["q_out"], "k": cache.k, "v": cache.v, "weights": cache.weights, "pos": cache.pos}
    if c["kind"] == "append4":
        B.dash_paged4_append(p, cache, s["k_new"], s["v_new"], s["row_start"], rotary=s["rotary"], q=s["q"], q_out=s["q_out"])
        B.dash_paged4_unpack(p, cache, s["k"], s["v"])
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    B.dash_paged4_attend(p, cache, s["q"], s["row_start"], s["o"], s["ws"], lse=s["lse"])
    return {"o": s["o"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"rotary": _rotary, "append_rot": _append_rot, "append4": _append4, "attend4": _attend4}[state["c"]["kind"]](state)


# ---- work ------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    lens, news = _lengths(c)
    es = 2 if c["dtype"] == "bf16" else 4
    h_q, h_kv, d = c["h_q"], c["h_kv"], c["d"]
    row, q_row = h_kv * d * es, h_q * d * es                     # a token's keys, or values; its queries
    row4 = h_kv * (d / 2 + d / 32)                               # keys, or values, in 4 bits
    if c["kind"] == "rotary":
        n = c["batch"] * c["len_hi"]
        return {"bytes": 2.0 * n * (row + q_row) + (4.0 * n if c["far"] else 0.0), "flops": 3.0 * n * (h_q + h_kv) * c["rot"]}
    if c["kind"] == "append_rot":
        return {"bytes": sum(news) * (4.0 * row + 2.0 * q_row + 8.0 * h_kv), "flops": 3.0 * sum(news) * (h_q + h_kv) * c["rot"]}
    if c["kind"] == "append4":
        pool = (sum(-(-n // c["page"]) for n in lens) + 3) * c["page"]
        return {"bytes": sum(news) * (2.0 * row + 2.0 * q_row + 2.0 * row4) + pool * 2.0 * (row4 + row), "flops": 3.0 * sum(news) * (h_q + h_kv) * c["rot"]}
    pairs = keys = rows = 0.0
    for n, m in zip(lens, news):
        rows += m
        pairs += m * n - (m * (m - 1) / 2 if c["causal"] else 0)
        keys += n
    return {"bytes": 2.0 * keys * row4 + rows * (2.0 * q_row + 4.0 * h_q), "flops": 4.0 * pairs * h_q * d}


# ---- the definitions in 64 bits, written apart from the plain forms -------------------------------------------------
def _exact_turn(c, x, pos):
    """Pairs as complex numbers, multiplied by mscale e^(i pos theta)."""
    rot = c["rot"]
    theta = []
    for i in range(rot // 2):
        base = c["base"]
        if c["scaling"] == "base":
            base *= c["factor"] ** (rot / (rot - 2))
        t = math.exp(-2.0 * i / rot * math.log(base))
        if c["scaling"] == "linear":
            t /= c["factor"]
        elif c["scaling"] == "parts":
            keep = min(max((ORIGINAL * t / (2 * math.pi) - LOW) / (HIGH - LOW), 0.0), 1.0)
            t = keep * t + (1 - keep) * t / c["factor"]
        theta.append(t)
    angle = pos.double()[..., None] * torch.tensor(theta, dtype=torch.float64, device=DEV)
    x = x.double()
    head, tail = x[..., :rot], x[..., rot:]
    pairs = head.unflatten(-1, (2, -1)).transpose(-1, -2) if c["layout"] == "halves" else head.unflatten(-1, (-1, 2))
    z = torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.full_like(angle, c["mscale"]), -angle if c["inverse"] else angle)
    pairs = torch.view_as_real(z)
    head = pairs.transpose(-1, -2).flatten(-2) if c["layout"] == "halves" else pairs.flatten(-2)
    return torch.cat((head, tail), -1)


def _exact_held(x):
    """What x [..., d] is held as in 4 bits: the nearest of the levels, the even one of two that are as near."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - 2)
    unit = torch.where(unit * 8 <= top, unit * 2, torch.where(unit * 4 > top, unit / 2, unit))   # log2 next to a power of two
    unit = torch.where(top > 7.25 * unit, 2 * unit, unit).clamp(2.0 ** -120, 2.0 ** 125)
    t = (b / unit).clamp(-6, 6)
    a = t.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.round(t / step) * step * unit).flatten(-2)     # round: half to even, and even multiples of a step are even codes


def _exact_unpacked(codes, scales):
    low, high = (codes & 15).int(), (codes >> 4).int()
    n = torch.stack((low, high), -1).flatten(-2)
    k, sign = n & 7, 1.0 - 2.0 * (n >> 3).double()
    mag = torch.where(k < 2, 0.5 * k.double(), (1.0 + 0.5 * (k & 1).double()) * torch.exp2((k >> 1).double() - 1.0))
    return sign * mag * torch.exp2(scales.double() - 127.0).repeat_interleave(32, -1)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "rotary":
        pos = s["pos"][:, None] if "pos" in s else torch.arange(c["len_hi"], device=DEV)
        return {"q": _exact_turn(c, s["q"], pos), "k": _exact_turn(c, s["k"], pos)}
    lens, news = _lengths(c)
    P, g, d = c["page"], c["h_q"] // c["h_kv"], c["d"]
    r0 = 0
    out = {}
    if c["kind"] == "attend4":
        out = {"o": torch.zeros((s["rows"], c["h_q"], d), dtype=torch.float64, device=DEV),
               "lse": torch.zeros((s["rows"], c["h_q"]), dtype=torch.float64, device=DEV)}
    else:
        pos = torch.cat([torch.arange(m, device=DEV) - m + int(s["seen"][b]) for b, m in enumerate(news)])
        out = {"q": _exact_turn(c, s["q"], pos[:, None])}
        k_new = _exact_turn(c, s["k_new"], pos[:, None])
        if c["kind"] == "append_rot":
            v_new = s["v_new"].double()
            out.update(k=s["k"].double(), v=s["v"].double(), weights=s["weights"].double(), pos=None)
        else:
            k_new, v_new = _exact_held(k_new), _exact_held(s["v_new"])
            out.update({name: _exact_unpacked(s[name + "_codes"], s[name + "_scales"]) for name in ("k", "v")})
    for b, (n, m) in enumerate(zip(lens, news)):
        at = torch.arange(n, device=DEV)
        page, off = s["table"][b].long()[at // P], at % P
        for h in range(c["h_kv"]):
            if c["kind"] != "attend4":
                p, o = page[n - m:], off[n - m:]
                out["k"][p, h, o], out["v"][p, h, o] = k_new[r0:r0 + m, h], v_new[r0:r0 + m, h]
                if "weights" in out:
                    out["weights"][p, h, o] = 0
                continue
            K, V = (_exact_unpacked(s[name + "_codes"][page, h, off], s[name + "_scales"][page, h, off]) for name in ("k", "v"))
            Q = s["q"][r0:r0 + m, h * g:(h + 1) * g].double().permute(1, 0, 2).reshape(g * m, d)
            x = torch.matmul(Q, K.t().contiguous()).view(g, m, n) / math.sqrt(d)
            if c["causal"]:
                x.masked_fill_(torch.ones((m, n), dtype=torch.bool, device=DEV).triu(n - m + 1), -math.inf)
            l = torch.logsumexp(x, -1)
            x = torch.exp(x - l[..., None]).view(g * m, n)
            out["o"][r0:r0 + m, h * g:(h + 1) * g] = torch.matmul(x, V).view(g, m, d).permute(1, 0, 2)
            out["lse"][r0:r0 + m, h * g:(h + 1) * g] = l.t()
            del x
        r0 += m
    return out
