"""What a serving runtime does with the KV blocks that this library swaps, as cases that can be timed and compared.

A cache is a pool of blocks as the library encrypts them: [block][K, V][token][kv head][channel] in 16 bits, a table of block
numbers for each request (-1: not on the device), a length for each request.

Operators ("op"), each a pass of a user's program
  append      a layer's new queries, keys and values out of their packed projection: norms per head, rotation, q returned, k and v
              written to their slots of the cache
  attend      one new token of each request over its blocks; "weigh": the blocks' accumulated attention weights are brought up to
              date; "keep": only over the blocks that a selection names for each kv head
  summarize   the bounds of the keys of blocks, in 8 bits
  select      the best blocks of each request and kv head by their bounds
  evict       the blocks with the least accumulated weight leave their tables

Fields of a case
  requests    requests of the batch (append: new tokens; summarize: blocks)
  tokens      the longest length of a request
  ragged      lengths (append, summarize: see there) spread below that one, one request empty; else all the same
  kv, group, dim, half
              kv heads, query heads to each, channels a head, "float16" or "bfloat16"
  block       tokens a block
  holes       share of the blocks that are not on the device
  weigh, keep, evict, rope
              as above; blocks that leave each request, at most; rotation's pairs: "halves" or "adjacent"
  mix         picks lengths and holes, so that every seed gives the same ones with other contents
"""
import math
import random

import torch

own = False

KEPT_FIRST, KEPT_LAST = 1, 2    # blocks at the ends of a request that are always selected, never evicted
DECAY = 0.9375
EPS = 1e-6


def _case(op, name=None, **fields):
    case = dict(op=op, requests=1, tokens=1, ragged=False, kv=8, group=4, dim=128, half="bfloat16", block=16, holes=0.0,
                weigh=False, keep=0, evict=0, rope="halves", mix=0)
    case.update(fields)
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # a first answer's first steps: one request of some tokens, 40 heads of 128, as in the library's swapped blocks
        _case("attend", "attend_one_short", tokens=33, kv=40, group=1, half="float16"),
        # a batch of conversations with the same heads, some blocks swapped out, weights kept for the next eviction
        _case("attend", "attend_batch_weigh", requests=32, tokens=2048, ragged=True, kv=40, group=1, half="float16",
              holes=0.08, weigh=True),
        # two long documents, grouped heads
        _case("attend", "attend_long", requests=2, tokens=131059, group=8),
        # long contexts of which each kv head reads 128 blocks
        _case("attend", "attend_selected", requests=16, tokens=65536, ragged=True, half="float16", keep=128),
        # a decode step of 64 requests
        _case("append", "append_decode", requests=64, tokens=4096, ragged=True),
        # a long prompt, 40 heads of 128
        _case("append", "append_prompt", requests=8191, tokens=8191, kv=40, group=1, half="float16"),
        # the blocks that a decode step wrote to
        _case("summarize", "summarize_decode", requests=64, ragged=True),
        # a whole long prompt's blocks
        _case("summarize", "summarize_prompt", requests=8192),
        # one long document: 256 of 8192 blocks
        _case("select", "select_one_long", tokens=131059, group=8, keep=256),
        # a batch of long contexts
        _case("select", "select_batch", requests=32, tokens=32768, ragged=True, keep=128),
        # room for one more block of one request
        _case("evict", "evict_one", tokens=2048, evict=1),
        # a batch of long contexts cut down
        _case("evict", "evict_batch", requests=256, tokens=131072, ragged=True, holes=0.3, evict=64),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _not_excluded(n):
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "summarize", "select", "evict"])
    kv, group = rng.choice([(40, 1), (32, 1), (8, 4), (8, 8), (4, 7), (2, 16), (1, 20), (5, 3)])
    dim = rng.choice([64, 80, 128, 128, 256])
    if kv * dim == 3072 or kv * group * dim == 3072:
        dim = 128
    fields = dict(kv=kv, group=group, dim=dim, half=rng.choice(["float16", "bfloat16"]), block=rng.choice([16, 16, 32, 64]),
                  ragged=rng.random() < 0.7, mix=rng.randrange(1 << 20))
    token = 4 * kv * dim    # bytes of one token's K and V
    if op == "attend":
        tokens = _not_excluded(_spread(rng, 1, 131072))
        most = max(1, min(128, (1 << 29) // (token * tokens)))
        fields.update(requests=_not_excluded(_spread(rng, 1, most)), tokens=min(tokens, (1 << 29) // token))
        kind = rng.randrange(3)
        if kind == 1:
            fields.update(weigh=True, holes=rng.choice([0.0, 0.1, 0.5]))
        if kind == 2:
            fields.update(keep=_spread(rng, 1, 256))
    elif op == "append":
        fields.update(requests=_not_excluded(_spread(rng, 1, min(8191, (1 << 28) // (token * (group + 2))))),
                      rope=rng.choice(["halves", "adjacent"]))
        fields.update(tokens=max(4096, fields["requests"]))
    elif op == "summarize":
        fields.update(requests=_not_excluded(_spread(rng, 1, min(8192, (1 << 28) // (token // 2 * fields["block"])))))
    elif op == "select":
        tokens = _not_excluded(_spread(rng, 1, 131072))
        blocks = -(-tokens // fields["block"])
        fields.update(requests=_not_excluded(_spread(rng, 1, max(1, min(64, (1 << 26) // (kv * dim * blocks))))),
                      tokens=tokens, keep=_spread(rng, 1, 512))
    else:
        fields.update(requests=_not_excluded(_spread(rng, 1, 256)), tokens=_not_excluded(_spread(rng, 1, 131072)),
                      holes=rng.choice([0.0, 0.3]), evict=_spread(rng, 1, 64))
    return _case(op, **fields)


# ---------------------------------------------------------------------------------------------
# shapes: what a case fixes whatever the seed

def _lengths(case):
    """tokens of each request"""
    rng = random.Random(case["mix"] * 7919 + 1)
    n, most = case["requests"], case["tokens"]
    if not case["ragged"]:
        return [most] * n
    got = [_spread(rng, max(1, most // 16), most) for _ in range(n)]
    got[0] = most
    if n > 2:
        got[n // 2] = 0
    return got


def _counts(case):
    """summarize: tokens of each block"""
    rng = random.Random(case["mix"] * 7919 + 2)
    return [rng.randint(1, case["block"]) if case["ragged"] else case["block"] for _ in range(case["requests"])]


def _blocks_of(case, tokens):
    return -(-tokens // case["block"])


def _holes(case):
    """for each request, whether each of its blocks is on the device"""
    rng = random.Random(case["mix"] * 7919 + 3)
    return [[rng.random() >= case["holes"] for _ in range(_blocks_of(case, n))] for n in _lengths(case)]


def work(case):
    kv, group, dim, bs = case["kv"], case["group"], case["dim"], case["block"]
    heads = kv * group
    if case["op"] == "append":
        n = case["requests"]
        elements = n * (heads + 2 * kv) * dim
        return {"bytes": 4 * elements + n * (4 * dim + 12) + 4 * dim, "flops": n * (heads + kv) * dim * 7}
    if case["op"] == "summarize":
        tokens = sum(_counts(case))
        return {"bytes": 2 * tokens * kv * dim + case["requests"] * (kv * (2 * dim + 4) + 8), "flops": 2 * tokens * kv * dim}
    lengths = _lengths(case)
    if case["op"] == "attend":
        n = case["requests"]
        if case["keep"]:
            tokens = sum(min(case["keep"] * bs, t) for t in lengths)
            tables = 4 * n * kv * case["keep"]
        else:
            tokens = sum(min(bs, t - j * bs) for t, there in zip(lengths, _holes(case)) for j, here in enumerate(there) if here)
            tables = 4 * sum(_blocks_of(case, t) for t in lengths) * (3 if case["weigh"] else 1)
        return {"bytes": 4 * tokens * kv * dim + 4 * n * heads * dim + 4 * n * heads + tables + 4 * n,
                "flops": 4 * tokens * heads * dim}
    blocks = sum(_blocks_of(case, t) for t in lengths)
    if case["op"] == "select":
        return {"bytes": blocks * (kv * (2 * dim + 4) + 4) + case["requests"] * (2 * heads * dim + kv * (4 * case["keep"] + 4)),
                "flops": 4 * blocks * heads * dim}
    return {"bytes": 12 * blocks + case["requests"] * (8 * case["evict"] + 8), "flops": blocks}


# ---------------------------------------------------------------------------------------------
# inputs

def _tables(case, g):
    """(tables [requests][most], lengths, blocks of the pool): the requests' blocks, in any order of the pool"""
    lengths, there = _lengths(case), _holes(case)
    most = max(1, max(_blocks_of(case, n) for n in lengths))
    here = torch.zeros(len(lengths), most, dtype=torch.bool)
    for i, row in enumerate(there):
        here[i, :len(row)] = torch.tensor(row, dtype=torch.bool)
    here = here.cuda()
    n = int(here.sum())
    tables = torch.full(here.shape, -1, dtype=torch.int32, device="cuda")
    tables[here] = torch.randperm(n + 3, generator=g, device="cuda")[:n].to(torch.int32)
    return tables, torch.tensor(lengths, dtype=torch.int32).cuda(), n + 3


def _pool(case, g, blocks):
    shape = (blocks, 2, case["block"], case["kv"], case["dim"])
    return torch.empty(shape, dtype=getattr(torch, case["half"]), device="cuda").normal_(generator=g)


def _some(blocks, most, rows, k, g):
    """for each request `rows` lists of k different blocks of its own, ascending, -1 where there are no more"""
    at = torch.rand(blocks.shape[0], rows, most, generator=g, device="cuda")
    at = at.masked_fill(torch.arange(most, device="cuda") >= blocks[:, None, None], 2.0)
    best, place = at.topk(min(k, most), dim=2, largest=False)
    place = place.masked_fill(best > 1.0, most).sort(dim=2).values
    return place.masked_fill(place == most, -1).to(torch.int32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + case["mix"])
    half, op = getattr(torch, case["half"]), case["op"]
    kv, dim, bs = case["kv"], case["dim"], case["block"]
    heads = kv * case["group"]
    s = {"case": case}

    def normal(*shape, dtype=half, std=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    if op == "append":
        n = case["requests"]
        # a prompt's tokens follow each other; a decode step's come one from each request
        decode = case["ragged"]
        if decode:
            at = torch.randint(0, case["tokens"], (n,), generator=g, device="cuda")
        else:
            at = torch.arange(n, device="cuda")
        blocks = max(256, _blocks_of(case, n) if not decode else n)
        order = torch.randperm(blocks, generator=g, device="cuda")
        block = order[torch.arange(n, device="cuda")] if decode else order[at // bs]
        angle = torch.arange(case["tokens"], device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
        packed = normal(n, (heads + 2 * kv) * dim)
        s.update(pool=_pool(case, g, blocks), q=packed[:, :heads * dim].unflatten(1, (heads, dim)),
                 k=packed[:, heads * dim:(heads + kv) * dim].unflatten(1, (kv, dim)),
                 v=packed[:, (heads + kv) * dim:].unflatten(1, (kv, dim)),
                 positions=at.to(torch.int32), slots=block * bs + at % bs,
                 q_weight=1 + normal(dim, std=0.2), k_weight=1 + normal(dim, std=0.2),
                 rope=torch.cat([angle.cos(), angle.sin()], 1).float(), q_out=torch.empty(n, heads, dim, dtype=half, device="cuda"))
    elif op == "summarize":
        n = case["requests"]
        blocks = torch.randperm(n + 3, generator=g, device="cuda")[:n].to(torch.int32)
        s.update(pool=_pool(case, g, n + 3), blocks=blocks, counts=torch.tensor(_counts(case), dtype=torch.int32).cuda(),
                 bounds=torch.zeros(n + 3, kv, 2, dim, dtype=torch.int8, device="cuda"),
                 scales=torch.zeros(n + 3, kv, dtype=torch.float32, device="cuda"))
    elif op == "attend":
        tables, lens, blocks = _tables(case, g)
        n = case["requests"]
        s.update(pool=_pool(case, g, blocks), tables=tables, lens=lens, q=normal(n, heads, dim, std=2.0),
                 out=torch.empty(n, heads, dim, dtype=half, device="cuda"), lse=torch.empty(n, heads, device="cuda"),
                 selected=_some((lens + bs - 1) // bs, tables.shape[1], kv, case["keep"], g) if case["keep"] else None)
        if case["weigh"]:
            kept = normal(*tables.shape, dtype=torch.float32).exp()
            s.update(kept=kept, weights=torch.empty_like(kept))
    elif op == "select":
        tables, lens, blocks = _tables(case, g)
        n = case["requests"]
        ends = torch.randint(-127, 128, (blocks, kv, 2, dim), generator=g, device="cuda", dtype=torch.int32)
        s.update(tables=tables, lens=lens, q=normal(n, heads, dim, std=2.0),
                 bounds=torch.stack([ends.amin(2), ends.amax(2)], 2).to(torch.int8),
                 scales=0.02 + 0.01 * torch.rand(blocks, kv, generator=g, device="cuda"),
                 selected=torch.empty(n, kv, case["keep"], dtype=torch.int32, device="cuda"),
                 counts=torch.empty(n, kv, dtype=torch.int32, device="cuda"))
    else:
        tables, lens, _ = _tables(case, g)
        n = case["requests"]
        s.update(tables=tables, lens=lens, weights=normal(*tables.shape, dtype=torch.float32, std=2.0).exp(),
                 evict=torch.randint(1, case["evict"] + 1, (n,), generator=g, device="cuda").to(torch.int32),
                 victims=torch.empty(n, case["evict"], dtype=torch.int32, device="cuda"),
                 victim_blocks=torch.empty(n, case["evict"], dtype=torch.int32, device="cuda"),
                 tables_out=torch.empty_like(tables))
    if "pool" in s:
        s.update(k_cache=s["pool"][:, 0], v_cache=s["pool"][:, 1])
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms

def _turn(x, weight, table, adjacent):
    """norm of each head, then rotation, in 32 bits"""
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    c, s = table.chunk(2, -1)
    c, s = c[:, None], s[:, None]
    if adjacent:
        u, v = x[..., 0::2], x[..., 1::2]
        return torch.stack([u * c - v * s, v * c + u * s], -1).flatten(-2)
    u, v = x.chunk(2, -1)
    return torch.cat([u * c - v * s, v * c + u * s], -1)


def _plain_append(s):
    adjacent, table, bs = s["case"]["rope"] == "adjacent", s["rope"][s["positions"].long()], s["case"]["block"]
    q = _turn(s["q"], s["q_weight"], table, adjacent).to(s["q"].dtype)
    k = _turn(s["k"], s["k_weight"], table, adjacent).to(s["k"].dtype)
    s["k_cache"][s["slots"] // bs, s["slots"] % bs] = k
    s["v_cache"][s["slots"] // bs, s["slots"] % bs] = s["v"]
    return {"q": q, "cache": s["pool"]}


def _plain_attend(s):
    case = s["case"]
    n, most = s["tables"].shape
    kv, group, dim, bs = case["kv"], case["group"], case["dim"], case["block"]
    at = s["selected"] if s["selected"] is not None else torch.arange(most, device="cuda", dtype=torch.int32).expand(n, kv, most)
    block = s["tables"].long()[:, None, :].expand(n, kv, most).gather(2, at.clamp(min=0).long())
    token = at[..., None] * bs + torch.arange(bs, device="cuda")
    valid = (at >= 0)[..., None] & (block >= 0)[..., None] & (token < s["lens"][:, None, None, None])
    block, head = block.clamp(min=0), torch.arange(kv, device="cuda")[None, :, None]
    k = s["k_cache"].transpose(1, 2)[block, head].float().flatten(2, 3)
    v = s["v_cache"].transpose(1, 2)[block, head].float()
    v = torch.where(valid[..., None], v, 0.0).flatten(2, 3)
    valid = valid.flatten(2)[:, :, None, :]
    logits = torch.matmul(s["q"].float().view(n, kv, group, dim) / math.sqrt(dim), k.transpose(2, 3).contiguous())
    logits = torch.where(valid, logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = (logits - top).exp()
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    got = {"out": torch.matmul(p, v).view(n, kv * group, dim).to(s["q"].dtype),
           "lse": (top + total.log()).view(n, kv * group)}
    if case["weigh"]:
        got["weights"] = DECAY * s["kept"] + p.view(n, kv * group, most, bs).sum((1, 3))
    return got


def _eighths(x, axis):
    """x in 8 bits, and the scale of each row: each step is defined with its rounding, so the whole numbers have one right value"""
    a = x.abs().amax(axis, keepdim=True)
    small = a < 1e-30
    full = torch.full_like(a, 127.0)
    q = torch.where(small, 0.0, torch.round(x * (full / torch.where(small, full, a))))
    return q, torch.where(small, 0.0, a / full)


def _plain_summarize(s):
    bs = s["case"]["block"]
    k = s["k_cache"][s["blocks"].long()].float()
    there = (torch.arange(bs, device="cuda") < s["counts"][:, None])[..., None, None]
    ends = torch.stack([torch.where(there, k, math.inf).amin(1), torch.where(there, k, -math.inf).amax(1)], 2)
    bounds, scales = _eighths(ends.flatten(2), -1)
    s["bounds"][s["blocks"].long()] = bounds.view_as(ends).to(torch.int8)
    s["scales"][s["blocks"].long()] = scales[..., 0]
    return {"bounds": s["bounds"], "scales": s["scales"]}


def _plain_select(s):
    case = s["case"]
    n, most = s["tables"].shape
    kv, group, dim, bs, keep = case["kv"], case["group"], case["dim"], case["block"], case["keep"]
    q, qs = _eighths(s["q"].float().view(n, kv, group, dim), -1)
    place = torch.arange(most, device="cuda")
    blocks = ((s["lens"] + bs - 1) // bs)[:, None]
    there = (place < blocks) & (s["tables"] >= 0)
    entry = s["tables"].clamp(min=0).long()
    low, high = s["bounds"][entry].permute(3, 0, 2, 4, 1).float()
    # whole numbers below 2^24: exact in any order
    total = torch.matmul(q.clamp(min=0), high.contiguous()) + torch.matmul(q.clamp(max=0), low.contiguous())
    score = (total * s["scales"][entry].transpose(1, 2)[:, :, None]) * qs
    score = score.amax(2) + 0.0
    always = there & ((place < KEPT_FIRST) | (place >= blocks - KEPT_LAST))
    score = torch.where(always[:, None], math.inf, torch.where(there[:, None], score, -math.inf))
    order = score.sort(dim=2, descending=True, stable=True).indices[..., :keep]
    count = there.sum(1).clamp(max=keep)[:, None].expand(n, kv)
    spare = torch.arange(order.shape[2], device="cuda") >= count[..., None]
    order = torch.where(spare, most, order).sort(dim=2).values
    s["selected"].fill_(-1)
    s["selected"][..., :order.shape[2]] = torch.where(order == most, -1, order)
    s["counts"].copy_(count)
    return {"selected": s["selected"], "counts": s["counts"]}


def _plain_evict(s):
    n, most = s["tables"].shape
    bs, m = s["case"]["block"], s["case"]["evict"]
    place = torch.arange(most, device="cuda")
    blocks = ((s["lens"] + bs - 1) // bs)[:, None]
    may = (place >= KEPT_FIRST) & (place < blocks - KEPT_LAST) & (s["tables"] >= 0)
    order = torch.where(may, s["weights"], math.inf).sort(dim=1, stable=True).indices[:, :m]
    count = torch.minimum(s["evict"].long(), may.sum(1))
    spare = torch.arange(order.shape[1], device="cuda") >= count[:, None]
    order = torch.where(spare, most, order).sort(dim=1).values
    spare = order == most
    s["victims"].fill_(-1)
    s["victim_blocks"].fill_(-1)
    s["victims"][:, :order.shape[1]] = torch.where(spare, -1, order)
    s["victim_blocks"][:, :order.shape[1]] = torch.where(spare, -1, s["tables"].gather(1, order.clamp(max=most - 1)))
    gone = torch.zeros(n, most + 1, dtype=torch.bool, device="cuda").scatter_(1, order, True)[:, :most]
    s["tables_out"].copy_(torch.where(gone, -1, s["tables"]))
    return {"victims": s["victims"], "blocks": s["victim_blocks"], "tables": s["tables_out"]}


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "summarize": _plain_summarize, "select": _plain_select,
          "evict": _plain_evict}


# ---------------------------------------------------------------------------------------------
# the framework's calls

def _own(s):
    import paper_2411_03357_amd as pgcm
    case = s["case"]
    op = case["op"]
    if "pool" in s and "cache" not in s:
        s["cache"] = pgcm.KVCache(s["k_cache"], s["v_cache"])
    if op == "append":
        pgcm.kv_append(s["cache"], s["q"], s["k"], s["v"], s["positions"], s["slots"], s["q_out"],
                       q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, rope=s["rope"],
                       adjacent=case["rope"] == "adjacent")
        return {"q": s["q_out"], "cache": s["pool"]}
    if op == "attend":
        pgcm.kv_attend(s["cache"], s["q"], s["tables"], s["lens"], s["out"], lse=s["lse"],
                       selected=s["selected"], weights=s.get("weights"), kept=s.get("kept"), decay=DECAY)
        got = {"out": s["out"], "lse": s["lse"]}
        if case["weigh"]:
            got["weights"] = s["weights"]
        return got
    if op == "summarize":
        pgcm.kv_summarize(s["cache"], s["blocks"], s["counts"], s["bounds"], s["scales"])
        return {"bounds": s["bounds"], "scales": s["scales"]}
    if op == "select":
        pgcm.kv_select(s["q"], s["tables"], s["lens"], s["bounds"], s["scales"], case["block"], s["selected"], s["counts"],
                       first=KEPT_FIRST, last=KEPT_LAST)
        return {"selected": s["selected"], "counts": s["counts"]}
    pgcm.kv_evict(s["weights"], s["tables"], s["lens"], case["block"], s["evict"], s["victims"], s["victim_blocks"],
                  s["tables_out"], first=KEPT_FIRST, last=KEPT_LAST)
    return {"victims": s["victims"], "blocks": s["victim_blocks"], "tables": s["tables_out"]}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_append(s):
    case, f = s["case"], torch.float64
    half = case["dim"] // 2

    def turned(x, w):
        x = x.to(f)
        x = x / ((x ** 2).sum(-1, keepdim=True) / case["dim"] + EPS) ** 0.5 * w.to(f)
        row = s["rope"].to(f)[s["positions"].long()][:, None]
        pairs = x.unflatten(-1, (half, 2)) if case["rope"] == "adjacent" else x.unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_complex(pairs.contiguous()) * torch.complex(row[..., :half], row[..., half:])
        z = torch.view_as_real(z)
        return (z if case["rope"] == "adjacent" else z.transpose(-1, -2)).flatten(-2)

    cache = s["pool"].to(f)
    rows = cache.transpose(1, 2).flatten(0, 1)      # [slot][K, V][head][channel]
    rows[s["slots"]] = torch.stack([turned(s["k"], s["k_weight"]), s["v"].to(f)], 1)
    cache = rows.view(cache.shape[0], case["block"], 2, case["kv"], case["dim"]).transpose(1, 2)
    return {"q": turned(s["q"], s["q_weight"]), "cache": cache}


def _exact_attend(s):
    case, f = s["case"], torch.float64
    kv, group, dim, bs = case["kv"], case["group"], case["dim"], case["block"]
    out = torch.zeros(case["requests"], kv * group, dim, dtype=f, device="cuda")
    lse = torch.full((case["requests"], kv * group), -math.inf, dtype=f, device="cuda")
    weights = DECAY * s["kept"].to(f) if case["weigh"] else None
    for b, n in enumerate(s["lens"].tolist()):
        for h in range(kv):
            places = torch.arange(_blocks_of(case, n), device="cuda") if s["selected"] is None else s["selected"][b, h].long()
            places = places[places >= 0]
            places = places[s["tables"][b, places] >= 0]
            token = (places[:, None] * bs + torch.arange(bs, device="cuda")).flatten()
            within = token < n
            if not bool(within.any()):
                continue
            block = s["tables"][b, places].long()
            k = s["k_cache"][block, :, h].to(f).flatten(0, 1)[within]
            v = s["v_cache"][block, :, h].to(f).flatten(0, 1)[within]
            mine = slice(h * group, (h + 1) * group)
            logits = (s["q"][b, mine].to(f) @ k.T) * dim ** -0.5
            lse[b, mine] = torch.logsumexp(logits, 1)
            p = (logits - lse[b, mine, None]).exp()
            out[b, mine] = p @ v
            if weights is not None:
                weights[b].index_add_(0, token[within] // bs, p.sum(0))
    got = {"out": out, "lse": lse}
    if weights is not None:
        got["weights"] = weights
    return got


def _exact_summarize(s):
    scales = s["scales"].to(torch.float64)
    k = s["k_cache"].to(torch.float64).abs()
    for block, count in zip(s["blocks"].tolist(), s["counts"].tolist()):
        scales[block] = k[block, :count].amax((0, 2)) / 127
    return {"bounds": None, "scales": scales}


def exact(case, seed):
    if case["op"] in ("select", "evict"):
        return None     # whole numbers alone
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "summarize": _exact_summarize}[case["op"]](s)
