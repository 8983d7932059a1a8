"""The calls of a serving loop over the 8-bit cache, as cases to time: appending K/V vectors, attention of one or several
query tokens, the attention weight that every cached token received, and eviction by it.

The cache holds e4m3 codes, row major [stream][token][d], and for every block of B tokens of a stream one scale 2^e: the
smallest power of two with max |x| <= 448 * 2^e.  A paged cache keeps its tokens in pages [page][kv head][token][d] behind a table
[sequence][logical page].  `states` [sequence][4] holds the length and the next position of every sequence.

A case is a dict of plain values:
  op        append    n vectors per stream behind the T (t_min .. T) that are there; ragged: counts from 1 to n
            attend    n query tokens per sequence (the last n of its T) over the cache
            weights   the softmax mass of those queries per cached token
            evict     down to `budget` tokens by weight, into another cache
  seqs, hkv, hq, d, B     sequences (layers x batch), KV heads, query heads, head dimension, tokens per scale
  page      tokens per page (0: contiguous)
  t_min     0: every sequence holds T vectors; else lengths drawn from [t_min, T]
  cap, window, slopes   cap * tanh(s / cap); positions further back than window are masked; distance bias per head
  bf16      16-bit type of queries, vectors and outputs
"""
import math
import random

import torch

own = False

_BASE = dict(op="attend", seqs=1, hkv=8, hq=32, d=128, B=64, page=0, T=4096, t_min=0, n=1, ragged=False, cap=0.0, window=0,
             slopes=False, bf16=False, budget=0, first=0, last=0)


def _case(**kw):
    return {**_BASE, **kw}


def listed():
    return [
        # one request on one layer, a short chat: the token of the step joins a block that is partly filled; latency counts
        _case(name="append_token", op="append", T=1100, n=1),
        # prefill of a long-context batch, four layers x 16 prompts of 8k tokens
        _case(name="append_prompts", op="append", seqs=64, T=0, n=8192, bf16=True),
        # continuous batching: 16 sequences of 96-channel heads get chunks of different, odd lengths on a paged cache
        _case(name="append_ragged", op="append", seqs=16, d=96, B=32, page=128, T=3000, t_min=1, n=2047, ragged=True),
        # one request on one layer, a short chat: the token's attention; latency and launches count
        _case(name="attend_token", T=1101),
        # a decode step over 16 sequences of 32k tokens
        _case(name="attend_long", seqs=16, T=32768, bf16=True),
        # a batch of unequal lengths, 256-channel heads, seven query heads per KV head, distance bias and a sliding window
        _case(name="attend_window", seqs=24, hkv=4, hq=28, d=256, B=128, T=16001, t_min=500, window=4096, slopes=True, bf16=True),
        # five draft tokens per sequence verified at once on a paged cache, capped scores
        _case(name="attend_drafts", seqs=32, B=32, page=256, T=6000, t_min=700, n=5, cap=50.0),
        # a chunk of a long prompt (chunked prefill) over the 16k tokens before and in it
        _case(name="attend_chunk", T=16384, n=1024, bf16=True),
        # the weights of one decode step over 16 sequences of 32k tokens
        _case(name="weights_step", op="weights", seqs=16, T=32768),
        # the last 32 tokens of a prompt observe the rest of it, on every layer of a 32-layer model; odd length
        _case(name="weights_window", op="weights", seqs=32, T=8191, n=32, bf16=True),
        # after the prefill of a 16k prompt on 32 layers: 1024 tokens are kept
        _case(name="evict_prompt", op="evict", seqs=32, T=16384, budget=1024, first=4, last=128),
        # a generation batch of unequal lengths, some under the budget
        _case(name="evict_batch", op="evict", seqs=64, hkv=2, hq=10, B=32, T=2300, t_min=600, budget=1600, first=0, last=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "weights", "weights", "evict", "evict"])
    hkv, r = rng.choice([(8, 4), (8, 4), (4, 7), (8, 1), (1, 8), (4, 8), (2, 5), (1, 16), (8, 2), (1, 24)])
    d = rng.choice([128, 128, 128, 64, 96, 256])
    c = _case(op=op, hkv=hkv, hq=hkv * r, d=d, B=rng.choice([32, 64, 64, 128]), page=rng.choice([0, 0, 0, 128, 256]), bf16=rng.random() < 0.5)
    c["seqs"] = _log_int(rng, 1, 64)
    if op == "append":
        c["n"] = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 8192)])
        c["T"] = rng.choice([0, _log_int(rng, 1, 8192)])
        c["ragged"] = c["n"] > 1 and rng.random() < 0.5
    else:
        c["T"] = _log_int(rng, 64, 32768)
        if op == "attend":
            c["n"] = rng.choice([1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 700)])
        elif op == "weights":
            c["n"] = rng.choice([1, 1, rng.randint(2, 40)])
        else:
            c["page"] = 0
            c["budget"] = max(1, int(c["T"] * rng.uniform(0.05, 0.9)))
            c["first"] = rng.choice([0, 0, min(4, c["budget"])])
            c["last"] = rng.choice([0, min(64, c["budget"] - c["first"])])
        if op in ("attend", "weights"):
            c["cap"] = rng.choice([0.0, 0.0, 0.0, 30.0])
            c["window"] = rng.choice([0, 0, 0, rng.randint(1, c["T"])])
            c["slopes"] = rng.random() < 0.25
            c["T"] = max(c["T"], c["n"])
    # no more than the largest listed case: vectors held and appended, and pairs of query rows and tokens
    while c["seqs"] > 1 and (c["seqs"] * hkv * d * max(c["T"], 1) > 2 ** 28 or c["seqs"] * hkv * d * c["n"] > 2 ** 28 or
                             c["seqs"] * hkv * r * c["n"] * max(c["T"], 1) > 2 ** 28):
        c["seqs"] //= 2
    if c["T"] > 3 and c["seqs"] > 1 and rng.random() < 0.4:
        c["t_min"] = max(c["n"] if op != "append" else 1, c["T"] // rng.randint(2, 20), 1)
    return c


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _capacity(case):
    t = case["T"] + (case["n"] if case["op"] == "append" else 0)
    unit = max(128, case["page"])
    return -(-t // unit) * unit


def _lengths(case, seed):
    r = random.Random(seed * 7919 + 17)
    lo = case["t_min"] or case["T"]
    length = [r.randint(lo, case["T"]) for _ in range(case["seqs"])]
    counts = [r.randint(1, case["n"]) if case["ragged"] else case["n"] for _ in range(case["seqs"])]
    return length, counts


def _vectors(case, gen, n, keys):
    """[seqs][n][hkv][d] in the 16-bit type, as a projection leaves them: keys with a few channels of larger spread and a mean
    of their own, values whose size differs from token to token."""
    dev, hkv, d = gen.device, case["hkv"], case["d"]
    x = torch.randn((case["seqs"], n, hkv, d), generator=gen, device=dev)
    if keys:
        spread = torch.where(torch.rand((hkv, d), generator=gen, device=dev) < 0.05, 4.0, 0.7)
        x = x.mul_(spread).add_(torch.randn((hkv, d), generator=gen, device=dev).mul_(spread))
    else:
        x = x.mul_(torch.exp(0.5 * torch.randn((case["seqs"], n, 1, 1), generator=gen, device=dev)))
    return x.to(torch.bfloat16 if case["bf16"] else torch.float16)


def _scale(amax):
    """The smallest power of two 2^e, e >= -126, with amax <= 448 * 2^e."""
    m, e = torch.frexp(amax)                 # amax = m * 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m > 0.875, e - 8, e - 9)
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e, -126).clamp(min=-126))


def _rows(case, table, cap):
    """[seqs][hkv][cap]: the row of the code arrays in which token t of a stream lives; then the row past the last one."""
    seqs, hkv, page = case["seqs"], case["hkv"], case["page"]
    t = torch.arange(cap, device=table.device)
    head = torch.arange(hkv, device=table.device)[None, :, None]
    if page:
        rows = (table.long()[:, t // page][:, None, :] * hkv + head) * page + (t % page)
        return rows, table.numel() * hkv * page
    return (torch.arange(seqs, device=table.device)[:, None, None] * hkv + head) * cap + t, seqs * hkv * cap


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    seqs, hkv, hq, d, B, op = (case[k] for k in ("seqs", "hkv", "hq", "d", "B", "op"))
    cap = _capacity(case)
    lens, counts = _lengths(case, seed)
    pages = cap // case["page"] if case["page"] else 1
    table = torch.randperm(seqs * pages, generator=gen, device=dev).to(torch.int32).view(seqs, pages)
    rows, n_rows = _rows(case, table, cap)
    s = {"case": case, "cap": cap, "table": table, "rows": rows, "n_rows": n_rows}
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["states"] = torch.stack([length, length, length * 0, length * 0], 1)
    # the arrays have a block of room at their end, which is not the cache's
    for name in ("k", "v"):
        codes = torch.zeros((n_rows + B, d), dtype=torch.uint8, device=dev)
        scale = torch.zeros(n_rows // B + 1, dtype=torch.float32, device=dev)
        if case["T"] > 0:
            x = torch.zeros((seqs, cap, hkv, d), dtype=torch.bfloat16 if case["bf16"] else torch.float16, device=dev)
            x[:, :case["T"]] = _vectors(case, gen, case["T"], name == "k")
            x *= (torch.arange(cap, device=dev) < length[:, None])[:, :, None, None]
            x = x.transpose(1, 2).reshape(seqs, hkv, cap // B, B, d)
            sc = _scale(x.abs().amax((3, 4)).float())
            codes[rows.reshape(-1)] = (x.float() / sc[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(-1, d)
            scale[rows[:, :, ::B].reshape(-1) // B] = sc.reshape(-1)
            del x
        s[name + "_codes"], s[name + "_scale"] = codes, scale
    s["pos"] = torch.arange(cap, dtype=torch.int32, device=dev).repeat(seqs, hkv, 1)
    # softmax masses: a few tokens hold most of it
    s["weight"] = torch.exp(2.0 * torch.randn((seqs, hkv, cap), generator=gen, device=dev))
    n = case["n"]
    if op == "append":
        s["k_new"], s["v_new"] = (_vectors(case, gen, n, keys).transpose(1, 2) for keys in (True, False))
        s["counts"] = torch.tensor(counts, dtype=torch.int32, device=dev) if case["ragged"] else None
        s["after"] = torch.zeros_like(s["states"])
    elif op in ("attend", "weights"):
        q = torch.randn((seqs, n, hq, d), generator=gen, device=dev).mul_(1.2)
        s["q"] = q.to(torch.bfloat16 if case["bf16"] else torch.float16).transpose(1, 2)
        s["scale"] = d ** -0.5
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, hq + 1, device=dev) / hq).float() if case["slopes"] else None
    if op == "weights":
        s["lse"] = _attention(s, values=False)[1]
        s["weight"].zero_()
    if op == "evict":
        s["to_cap"] = -(-case["budget"] // 128) * 128
        for name in ("k", "v"):
            s["to_%s_codes" % name] = torch.zeros((seqs * hkv * s["to_cap"], d), dtype=torch.uint8, device=dev)
            s["to_%s_scale" % name] = torch.zeros(seqs * hkv * s["to_cap"] // B, device=dev)
        s["to_pos"] = torch.zeros((seqs, hkv, s["to_cap"]), dtype=torch.int32, device=dev)
        s["to_weight"] = torch.zeros((seqs, hkv, s["to_cap"]), device=dev)
        s["after"] = torch.zeros_like(s["states"])
    if own:
        from paper_2510_05176_amd import patternkv as pk
        kw = dict(n_seq=seqs, n_kv_heads=hkv, n_q_heads=hq, head_dim=d, block=B, dtype=pk.DTYPE_BF16 if case["bf16"] else pk.DTYPE_FP16)
        s["cfg"] = pk.Fp8Config(t_capacity=cap, page_tokens=case["page"], n_pages=seqs * pages if case["page"] else 0, **kw)
        s["cache"] = pk.Fp8Cache(s["cfg"], arrays={k: s[k] for k in ("k_codes", "v_codes", "k_scale", "v_scale", "pos", "weight")},
                                 states=s["states"], page_table=table if case["page"] else None)
        if op == "evict":
            s["to_cfg"] = pk.Fp8Config(t_capacity=s["to_cap"], **kw)
            s["to"] = pk.Fp8Cache(s["to_cfg"], arrays={k: s["to_" + k] for k in ("k_codes", "v_codes", "k_scale", "v_scale", "pos", "weight")},
                                  states=s["after"])
    return s


# ---- the plain form ----------------------------------------------------------------------------------------------------------

def _held(s, name):
    """What the cache's codes stand for, [seqs][hkv][cap][d] in 32 bits."""
    B = s["case"]["B"]
    x = s[name + "_codes"][s["rows"]].view(torch.float8_e4m3fn).float()
    return x.unflatten(2, (-1, B)).mul_(s[name + "_scale"][s["rows"][:, :, ::B] // B][..., None, None]).flatten(2, 3)


def _append(s):
    case = s["case"]
    seqs, hkv, d, B, n, cap = case["seqs"], case["hkv"], case["d"], case["B"], case["n"], s["cap"]
    dev = s["rows"].device
    length, nxt = s["states"][:, 0].long(), s["states"][:, 1].long()
    count = s["counts"].long() if s["counts"] is not None else torch.full_like(length, n)
    blocks = (n + B - 2) // B + 1                                                # as many as n vectors can touch
    t = length[:, None] // B * B + torch.arange(blocks * B, device=dev)
    new = (t >= length[:, None]) & (t < length[:, None] + count[:, None])
    live = t < length[:, None] + count[:, None]
    rows = torch.where(live[:, None], s["rows"].gather(2, t.clamp(max=cap - 1)[:, None].expand(-1, hkv, -1)), s["n_rows"])
    first = s["rows"].gather(2, t[:, None, :B].clamp(max=cap - 1).expand(-1, hkv, -1))
    partly = (length % B > 0)[:, None]
    at = (t - length[:, None]).clamp(0, n - 1)[:, None, :, None].expand(-1, hkv, -1, d)
    for name in ("k", "v"):
        codes, scale = s[name + "_codes"], s[name + "_scale"]
        x = s[name + "_new"].gather(2, at).float() * new[:, None, :, None]
        was = scale[first[:, :, 0] // B]
        x[:, :, :B] += codes[first].view(torch.float8_e4m3fn).float().nan_to_num(0.0) * was[..., None, None] * (t[:, None, :B, None] < length[:, None, None, None])
        x = x.unflatten(2, (blocks, B))
        amax = (x * new.view(seqs, 1, blocks, B, 1)).abs().amax((3, 4))
        sc = _scale(amax)
        sc[:, :, 0] = torch.where(partly, torch.maximum(sc[:, :, 0], was), sc[:, :, 0])
        codes[rows] = (x / sc[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).flatten(2, 3)
        # blocks that got none keep their scale
        got = (new.view(seqs, blocks, B).any(2))[:, None].expand(-1, hkv, -1)
        scale[torch.where(got, s["rows"].gather(2, t[:, None, ::B].clamp(max=cap - 1).expand(-1, hkv, -1)), s["n_rows"]) // B] = sc
    wide = torch.cat([s["pos"], s["pos"][:, :, :1]], 2)
    to = torch.where(new, t, cap)[:, None].expand(-1, hkv, -1)
    s["pos"].copy_(wide.scatter_(2, to, (nxt[:, None] + t - length[:, None]).int()[:, None].expand(-1, hkv, -1))[:, :, :cap])
    s["weight"].copy_(torch.cat([s["weight"], s["weight"][:, :, :1]], 2).scatter_(2, to, 0.0)[:, :, :cap])
    s["after"].copy_(torch.stack([length + count, nxt + count, count * 0, count * 0], 1))


def _appended(s):
    n, B = s["n_rows"], s["case"]["B"]
    return {"k_codes": s["k_codes"][:n].view(torch.float8_e4m3fn), "v_codes": s["v_codes"][:n].view(torch.float8_e4m3fn),
            "k_scale": s["k_scale"][:n // B], "v_scale": s["v_scale"][:n // B], "pos": s["pos"], "weight": s["weight"], "states": s["after"]}


def _scores(s):
    """[seqs][hkv][n * r][cap] scaled, capped and biased scores, masked ones at -inf; the query's token is the slower index."""
    case = s["case"]
    seqs, hkv, hq, n, cap = case["seqs"], case["hkv"], case["hq"], case["n"], s["cap"]
    r, dev = hq // hkv, s["rows"].device
    q = s["q"].float().unflatten(1, (hkv, r)).transpose(2, 3).flatten(2, 3)
    x = torch.matmul(q, _held(s, "k").transpose(2, 3)).mul_(s["scale"])
    if case["cap"]:
        x = torch.tanh(x / case["cap"]).mul_(case["cap"])
    length, nxt = s["states"][:, 0], s["states"][:, 1]
    i = torch.arange(n, device=dev)
    x = x.unflatten(2, (n, r))
    seen = (torch.arange(cap, device=dev) <= (length[:, None] - n + i)[..., None])[:, None]
    if case["window"] or case["slopes"]:
        back = (nxt[:, None] - n + i)[:, None, :, None] - s["pos"][:, :, None, :]
        if case["slopes"]:
            x = x - s["slopes"].view(1, hkv, 1, r, 1) * back[:, :, :, None].float()
        if case["window"]:
            seen = seen & (back < case["window"])
    return x.masked_fill(~seen[:, :, :, None], -math.inf).flatten(2, 3)


def _attention(s, values=True):
    case = s["case"]
    x = _scores(s)
    most = x.amax(3, keepdim=True)
    x = torch.exp(x.sub_(most.masked_fill(most == -math.inf, 0.0)))
    mass = x.sum(3, keepdim=True)
    back = lambda y: y.unflatten(2, (case["n"], -1)).transpose(2, 3).flatten(1, 2)   # noqa: E731  [seqs][hq][n]...
    lse = back((most + torch.log(mass))[..., 0])
    if not values:
        return None, lse
    v = _held(s, "v")
    o = torch.matmul(x, v) / mass.masked_fill(mass == 0, 1.0)
    return back(o).to(s["q"].dtype), lse


def _weights(s):
    case = s["case"]
    lse = s["lse"].unflatten(1, (case["hkv"], -1)).transpose(2, 3).flatten(2, 3)[..., None]
    w = torch.exp(_scores(s).sub_(lse.masked_fill(lse == -math.inf, 0.0))).sum(2)
    live = (torch.arange(s["cap"], device=w.device) < s["states"][:, :1])[:, None]
    s["weight"].copy_(torch.where(live, w, s["weight"]))


def _evict(s):
    case = s["case"]
    seqs, hkv, d, B, cap, budget, to_cap = case["seqs"], case["hkv"], case["d"], case["B"], s["cap"], case["budget"], s["to_cap"]
    dev = s["rows"].device
    length = s["states"][:, 0].long()[:, None, None]
    t = torch.arange(cap, device=dev)
    always = (t < case["first"]) | (t >= length - case["last"])
    key = torch.where(t < length, torch.where(always, math.inf, s["weight"]), -math.inf)
    keep = key.sort(dim=2, descending=True, stable=True).indices[:, :, :budget].sort(dim=2).values
    live = torch.arange(budget, device=dev) < length.clamp(max=budget)
    rows = s["rows"].gather(2, keep)
    room = torch.nn.functional.pad(live.expand(-1, hkv, -1), (0, to_cap - budget))
    for name in ("k", "v"):
        x = s[name + "_codes"][rows].view(torch.float8_e4m3fn).float() * s[name + "_scale"][rows // B][..., None]
        x = torch.nn.functional.pad(x.masked_fill(~live[..., None], 0.0), (0, 0, 0, to_cap - budget)).unflatten(2, (-1, B))
        sc = _scale(x.abs().amax((3, 4)))
        codes = (x / sc[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).flatten(2, 3)
        old = s["to_%s_codes" % name].view(seqs, hkv, to_cap, d)
        old.copy_(torch.where(room[..., None], codes, old))
        old = s["to_%s_scale" % name].view(seqs, hkv, -1)
        old.copy_(torch.where(room[:, :, ::B], sc, old))
    for name in ("pos", "weight"):
        old = s["to_" + name][:, :, :budget]
        old.copy_(torch.where(live, s[name].gather(2, keep), old))
    s["after"].copy_(torch.cat([s["states"][:, :1].clamp(max=budget), s["states"][:, 1:2], s["states"][:, 2:] * 0], 1))


def _evicted(s):
    return {"k_codes": s["to_k_codes"].view(torch.float8_e4m3fn), "v_codes": s["to_v_codes"].view(torch.float8_e4m3fn),
            "k_scale": s["to_k_scale"], "v_scale": s["to_v_scale"], "pos": s["to_pos"], "weight": s["to_weight"], "states": s["after"]}


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2510_05176_amd import patternkv as pk
        if op == "append":
            pk.pk_fp8_append(s["cfg"], s["cache"], s["k_new"], s["v_new"], counts=s["counts"], states_out=s["after"])
            return _appended(s)
        if op == "evict":
            pk.pk_fp8_evict(s["cfg"], s["cache"], s["to_cfg"], s["to"], case["budget"], keep_first=case["first"], keep_last=case["last"])
            return _evicted(s)
        how = dict(cap=case["cap"], window=case["window"], slopes=s["slopes"])
        if op == "attend":
            lse = torch.empty(s["q"].shape[:3], device=s["q"].device)
            return {"out": pk.pk_fp8_attention(s["cfg"], s["cache"], s["q"], s["scale"], lse=lse, **how), "lse": lse}
        pk.pk_fp8_weights(s["cfg"], s["cache"], s["q"], s["lse"], s["scale"], accumulate=False, **how)
        return {"weight": s["weight"]}
    if op == "append":
        _append(s)
        return _appended(s)
    if op == "evict":
        _evict(s)
        return _evicted(s)
    if op == "attend":
        out, lse = _attention(s)
        return {"out": out, "lse": lse}
    _weights(s)
    return {"weight": s["weight"]}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------

def work(case):
    # lengths of unequal sequences: their mean; a cached token is a row of codes in K and V, a share of two scales, in the passes
    # that need it its position
    hkv, d, B, n, op = case["hkv"], case["d"], case["B"], case["n"], case["op"]
    length = ((case["t_min"] + case["T"]) / 2 if case["t_min"] else case["T"])
    streams = case["seqs"] * hkv
    row = d + 4 / B
    if op == "append":
        new = streams * ((n + 1) / 2 if case["ragged"] else n)
        return {"bytes": new * (2 * 2 * d + 2 * row + 8), "flops": new * 2 * d}
    if op == "evict":
        kept = streams * min(length, case["budget"])
        return {"bytes": streams * length * 4 + kept * 2 * (2 * row + 8), "flops": kept * 2 * d}
    queries = case["seqs"] * case["hq"] * n
    seen = min(length - (n - 1) / 2, case["window"]) if case["window"] else length - (n - 1) / 2
    read = min(length, seen + n - 1)
    pos = 4 if case["window"] or case["slopes"] else 0
    if op == "weights":
        return {"bytes": streams * read * (row + pos) + streams * length * 4 + queries * (2 * d + 4), "flops": queries * seen * (2 * d + 4)}
    return {"bytes": streams * read * (2 * row + pos) + queries * (4 * d + 4), "flops": queries * seen * (4 * d + 6)}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------

def _value_e4m3(byte):
    """What an e4m3 byte stands for: sign, four bits of exponent (bias 7), three of mantissa; no infinities."""
    b = byte.long()
    sign, e, m = 1.0 - 2.0 * (b >> 7).double(), (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1.0 + m / 8.0) * torch.exp2((e - 7).double()))
    return sign * v


def _nearest_e4m3(x):
    """The nearest e4m3 value of x, |x| <= 448, ties to even: steps of 2^-3 of the power of two below, of 2^-9 under 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(x / step) * step


def _block_scale(x):
    """[..., B, d] -> the block's scale, by trying the powers of two around the quotient."""
    amax = x.abs().flatten(-2).amax(-1)
    e = torch.floor(torch.log2((amax / 448.0).clamp(min=2.0 ** -126))) - 1.0
    for _ in range(3):
        e = torch.where(amax > 448.0 * torch.exp2(e), e + 1.0, e)
    return torch.exp2(e.clamp(min=-126.0))


def exact(case, seed):
    s = prepare(case, seed)
    op, seqs, hkv, hq, d, B, n = (case[k] for k in ("op", "seqs", "hkv", "hq", "d", "B", "n"))
    cap = s["cap"]
    r, rows = hq // hkv, s["rows"]
    lens = s["states"][:, 0].tolist()

    def held(name, b):
        x = _value_e4m3(s[name + "_codes"][rows[b]])
        return (x.view(hkv, cap // B, B, d) * s[name + "_scale"].double()[rows[b][:, ::B] // B][..., None, None]).view(hkv, cap, d)

    if op == "append":
        counts = s["counts"].tolist() if s["counts"] is not None else [n] * seqs
        got = {}
        for name in ("k", "v"):
            codes = torch.empty((s["n_rows"], d), dtype=torch.float64, device=rows.device)
            scale = s[name + "_scale"].double()[:s["n_rows"] // B]
            for b in range(seqs):
                old = _value_e4m3(s[name + "_codes"][rows[b]]).view(hkv, cap // B, B, d)
                was = scale[rows[b][:, ::B] // B].clone()
                end = lens[b] + counts[b]
                lo, hi = lens[b] // B, -(-end // B)
                x = torch.zeros((hkv, (hi - lo) * B, d), dtype=torch.float64, device=rows.device)
                keep = lens[b] - lo * B
                x[:, keep:end - lo * B] = s[name + "_new"][b, :, :counts[b]].double()
                x = x.view(hkv, hi - lo, B, d)
                sc = _block_scale(x)
                if keep:
                    sc[:, 0] = torch.maximum(sc[:, 0], was[:, lo])
                    x[:, 0, :keep] = old[:, lo, :keep] * was[:, lo, None, None]
                fresh = _nearest_e4m3(x / sc[..., None, None]).view(hkv, -1, d)
                all_codes = old.reshape(hkv, cap, d)
                all_codes[:, lo * B:end] = fresh[:, :end - lo * B]
                was[:, lo:hi] = sc
                codes[rows[b].reshape(-1)] = all_codes.reshape(-1, d)
                scale[rows[b][:, ::B].reshape(-1) // B] = was.reshape(-1)
            got[name + "_codes"], got[name + "_scale"] = codes, scale
        # whole numbers, and the weights (zero where a vector is new), have no rounding to look at
        return {**got, "pos": None, "weight": None, "states": None}
    if op == "evict":
        got = {"weight": torch.zeros((seqs, hkv, s["to_cap"]), dtype=torch.float64, device=rows.device)}
        for name in ("k", "v"):
            got[name + "_codes"] = torch.zeros((seqs, hkv, s["to_cap"], d), dtype=torch.float64, device=rows.device)
            got[name + "_scale"] = torch.zeros((seqs, hkv, s["to_cap"] // B), dtype=torch.float64, device=rows.device)
        for b in range(seqs):
            length, new = lens[b], min(lens[b], case["budget"])
            w = s["weight"][b, :, :length].double().clone()
            w[:, :case["first"]] = math.inf
            w[:, length - case["last"]:] = math.inf
            order = torch.argsort(-w, dim=1, stable=True)[:, :new].sort(dim=1).values
            got["weight"][b, :, :new] = s["weight"][b].double().gather(1, order)
            nb = -(-new // B)
            for name in ("k", "v"):
                x = torch.zeros((hkv, nb * B, d), dtype=torch.float64, device=rows.device)
                x[:, :new] = held(name, b).gather(1, order[..., None].expand(-1, -1, d))
                x = x.view(hkv, nb, B, d)
                sc = _block_scale(x)
                got[name + "_scale"][b, :, :nb] = sc
                got[name + "_codes"][b, :, :new] = _nearest_e4m3(x / sc[..., None, None]).view(hkv, -1, d)[:, :new]
        got = {k: v.view(-1, d) if k.endswith("codes") else v.view(-1) if k.endswith("scale") else v for k, v in got.items()}
        return {**got, "pos": None, "states": None}
    outs, lses, masses = [], [], []
    for b in range(seqs):
        length, first = lens[b], int(s["states"][b, 1]) - n
        q = s["q"][b].double().view(hkv, r, n, d)
        x = torch.matmul(q.reshape(hkv, r * n, d), held("k", b)[:, :length].transpose(1, 2)).view(hkv, r, n, length) * s["scale"]
        if case["cap"]:
            x = case["cap"] * torch.tanh(x / case["cap"])
        place = first + torch.arange(n, device=rows.device)
        dist = place[None, :, None] - s["pos"][b, :, None, :length].long()
        if case["slopes"]:
            x = x - s["slopes"].double().view(hkv, r, 1, 1) * dist[:, None].double()
        hidden = torch.arange(length, device=rows.device) > (length - n + torch.arange(n, device=rows.device))[:, None]
        hidden = hidden.expand(hkv, n, length)
        if case["window"]:
            hidden = hidden | (dist >= case["window"])
        x = x.masked_fill(hidden[:, None], -math.inf)
        lse = torch.logsumexp(x, 3)
        if op == "weights":
            p = torch.exp(x - s["lse"][b].double().view(hkv, r, n, 1))
            w = s["weight"][b].double()
            w[:, :length] = p.sum((1, 2))
            masses.append(w)
            continue
        p = torch.exp(x - lse[..., None])
        outs.append(torch.matmul(p.view(hkv, r * n, length), held("v", b)[:, :length]).view(hq, n, d))
        lses.append(lse.view(hq, n))
    if op == "weights":
        return {"weight": torch.stack(masses)}
    return {"out": torch.stack(outs), "lse": torch.stack(lses)}
