"""Choosing what to read and what to keep of the engine's KV pool, with the sizes the operators are measured at.

bounds:  how far the keys of every block that has become full reach in each channel, in 8 bits.
select:  for each new token and KV head the blocks whose keys can score highest with its queries, by those bounds.
sparse:  attention of the new tokens over the selected blocks alone.
weigh:   attention weight that every block of a sequence gets from the new tokens, added to what it had.
evict:   a sequence's blocks of least weight leave its table.

A batch holds `seqs` sequences. Sequence s brings new[s] tokens on top of past[s] cached ones; its 16-token blocks lie
in arbitrary slots of the pool, listed in its row of the block table. `own` chooses between the plain torch form and
the engine's kernels.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(op, name=None, **kw):
    c = dict(op=op, dtype="bf16", layout=0, kv_heads=8, group=4, head_dim=128, seqs=1, new_lo=1, new_hi=1, past_lo=0,
             past_hi=0, mix=1)
    if op in ("select", "sparse", "evict"):
        c.update(budget=64, first=1, last=2)
    if op == "sparse":
        c.update(lse=False)
    if op == "weigh":
        c.update(window=0, keep=1.0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step of 32 sessions that brings a few accepted tokens each: some fill a block; all launch latency
        _case("bounds", "bounds step 32", seqs=32, new_lo=1, new_hi=7, past_lo=100, past_hi=8000),
        # a long session's blocks are back in the pool: all its bounds are made again
        _case("bounds", "bounds prefix 130k", new_lo=130500, new_hi=130500),
        # one new token of one long agent session (258 K tokens)
        _case("select", "select step 1 x 258k", past_lo=258047, past_hi=258047),
        # a chunk of new tokens (a tool result) at the end of a long session
        _case("select", "select chunk 500 x 128k", new_lo=500, new_hi=500, past_lo=130500, past_hi=130500),
        # one new token of one session, whatever its length: latency
        _case("sparse", "sparse step 1", past_lo=258047, past_hi=258047),
        # one new token each of 32 sessions of very different lengths, wide groups, a large budget
        _case("sparse", "sparse step 32 ragged", seqs=32, group=12, past_lo=2000, past_hi=130000, budget=256, mix=2, lse=True),
        # several sessions bring tool results of odd lengths, fp16, block-major
        _case("sparse", "sparse chunks ragged", dtype="fp16", layout=1, seqs=7, new_lo=33, new_hi=500, past_lo=500,
              past_hi=70000, mix=4),
        # one new token of one short session: latency
        _case("weigh", "weigh step 1 x 1k", past_lo=1000, past_hi=1000),
        # one new token each of 32 sessions of very different lengths, wide groups
        _case("weigh", "weigh step 32 ragged", seqs=32, group=12, past_lo=2000, past_hi=130000, mix=2),
        # prefill of one 8 K prompt
        _case("weigh", "weigh prompt 8k", new_lo=8192, new_hi=8192),
        # one session is cut down
        _case("evict", "evict 1 x 16k", past_lo=16000, past_hi=16000, budget=512),
        # 32 sessions of very different lengths, some of them below the budget
        _case("evict", "evict 32 ragged", seqs=32, past_lo=2000, past_hi=250000, budget=1000, first=4, last=32, mix=2),
    ]


def _between(rng, lo, hi):
    """Whole number in [lo, hi], spread over its logarithm."""
    return min(hi, int((lo + 1) * math.exp(rng.random() * math.log((hi + 1.999) / (lo + 1)))) - 1)


def draw(rng):
    """A case of the same ranges: whichever operator, 1 .. 64 sequences, prompts from one token up."""
    op = rng.choice(["bounds", "select", "sparse", "weigh", "evict"])
    heads, head_dim = rng.choice([(2, 64), (4, 64), (4, 128), (8, 128), (1, 128)])
    c = dict(dtype=rng.choice(["bf16", "fp16"]), layout=rng.randrange(2), kv_heads=heads, head_dim=head_dim,
             group=rng.choice([1, 2, 3, 4, 7, 8, 12]), mix=rng.randrange(1 << 20))
    if op == "bounds":
        total = _between(rng, 20, 120000)
        seqs = _between(rng, 1, min(total, 64))
        new = -(-total // seqs)
        return _case(op, seqs=seqs, new_lo=_between(rng, 1, new), new_hi=new, past_hi=_between(rng, 0, 100000 // seqs), **c)
    if op == "evict":
        total = _between(rng, 200, 1200000)
        seqs = _between(rng, 1, min(64, total // 100))
        hi = min(250000, total // seqs + 1)
        budget = _between(rng, 3, max(4, hi // 32))
        first = rng.randrange(0, min(budget - 1, 5))
        return _case(op, seqs=seqs, past_lo=_between(rng, hi // 4, hi), past_hi=hi, budget=budget, first=first,
                     last=_between(rng, 1, budget - first - 1), **c)
    more = {}
    if op != "weigh":
        budget = _between(rng, 3, 256)
        first = rng.randrange(0, min(budget - 1, 3))
        more = dict(budget=budget, first=first, last=_between(rng, 1, max(1, min(8, budget - first - 1))))
    if op == "sparse":
        more["lse"] = rng.random() < 0.5
    if op == "weigh":
        more = dict(window=rng.choice([0, 0, 0, _between(rng, 16, 4096)]), keep=rng.choice([1.0, 1.0, 0.9]))
    c.update(more)
    least = BLOCK * (budget + 2) if op == "select" else 0       # there is something to choose from
    if rng.random() < 0.5:      # one new token each
        total = _between(rng, 3000, 1200000)
        seqs = _between(rng, 1, 64)
        hi = max(least, min(250000, total // seqs + 1))
        return _case(op, seqs=seqs, past_lo=_between(rng, least, hi), past_hi=hi, **c)
    # prompts and chunks
    rows = heads * c["group"]
    most = {"select": 2000, "sparse": min(2000, 90000 // c.get("budget", 1)), "weigh": int((1.5e9 / rows) ** 0.5)}[op]
    total = _between(rng, 10, most)
    seqs = _between(rng, 1, 8)
    new = total // seqs + 1
    most = int((7e8 / rows if op == "weigh" else 2.4e7) / (total + 500) / seqs)
    past = max(least, _between(rng, most // 30, most))
    return _case(op, seqs=seqs, new_lo=_between(rng, 1, new), new_hi=new, past_lo=least, past_hi=past, **c)


def _lengths(case):
    """New and cached tokens of every sequence; they belong to the case, not to the seed."""
    rng = random.Random(case["mix"])
    pick = lambda lo, hi: _between(rng, min(lo, hi), hi)  # noqa: E731
    new, past = ([pick(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])],
                 [pick(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])])
    if case["op"] == "bounds":      # the first one's last token fills a block
        past[0] += -(past[0] + new[0]) % BLOCK
    return new, past


def work(case):
    c = case
    h, d, g = c["kv_heads"], c["head_dim"], c["group"]
    new, past = _lengths(c)
    t = sum(new)
    if c["op"] == "bounds":     # keys of the blocks that become full, two bytes a channel and one a head
        full = sum((n + p) // BLOCK - p // BLOCK for n, p in zip(new, past))
        return {"bytes": full * h * (2 * BLOCK * d + 2 * d + 1), "flops": 2 * full * BLOCK * h * d}
    if c["op"] == "evict":      # slots and weights read, slots and weights or evicted slots written
        blocks = sum(-(-(n + p) // BLOCK) for n, p in zip(new, past))
        return {"bytes": 16 * blocks, "flops": blocks}
    q = 2 * t * h * g * d
    if c["op"] == "select":     # the bounds of the blocks in front of the last query's own
        blocks = sum((n + p - 1) // BLOCK for n, p in zip(new, past))
        pairs = sum(sum((p + i) // BLOCK for i in range(n)) for n, p in zip(new, past))
        return {"bytes": q + blocks * h * (2 * d + 1) + 4 * t * h * c["budget"], "flops": 4 * pairs * h * d}
    if c["op"] == "sparse":     # every block that is selected at least once: all, or as many as the tokens can name
        seen = [[min(c["budget"], (p + i) // BLOCK + 1) for i in range(n)] for n, p in zip(new, past)]
        blocks = sum(min(sum(s), -(-(n + p) // BLOCK)) for s, n, p in zip(seen, new, past))
        pairs = BLOCK * sum(sum(s) for s in seen)
        return {"bytes": blocks * h * 2 * BLOCK * d * 2 + 2 * q + 4 * t * h * c["budget"] + (4 * t * h * g if c["lse"] else 0),
                "flops": 4 * pairs * h * g * d}
    pairs = keys = 0
    for n, p in zip(new, past):
        w = c["window"] or n + p
        pairs += int(np.minimum(np.arange(p + 1, p + n + 1, dtype=np.int64), w).sum())
        keys += min(n + p, w + n - 1)
    return {"bytes": 2 * keys * h * d + q + 4 * t * h * g + 8 * sum(-(-(n + p) // BLOCK) for n, p in zip(new, past)),
            "flops": 2 * pairs * h * g * d}


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(dev).manual_seed(seed * 1000003 + 29)
    dt = DTYPES[c["dtype"]]
    new, past = _lengths(c)
    kv = [n + p for n, p in zip(new, past)]
    blocks = [-(-n // BLOCK) for n in kv]
    n_slots = sum(blocks) + 3 + sum(blocks) // 50
    h, d, g, op = c["kv_heads"], c["head_dim"], c["group"], c["op"]
    s = {"case": c}
    held = 1 if op in ("select", "evict") else n_slots      # these two do not read the pool
    if own:
        from paper_2609_39819_b200 import binding
        s["engine"] = binding.Engine(n_layers=1, n_kv_heads=h, head_dim=d, pool_layout=c["layout"], n_hbm_blocks=n_slots,
                                     n_host_blocks=0, max_contexts=1, max_messages=16, max_tokens=64, zero_pools=False)
        pool = s["engine"].hbm_pool.view(dt)
    else:
        pool = torch.empty(2 * held * BLOCK * h * d, dtype=dt, device=dev)
    if held > 1:
        pool.normal_(generator=gen)
        # K and V as [slot, token, head, dim]
        pool = pool.view(2, n_slots, BLOCK, h, d) if c["layout"] == 0 else pool.view(n_slots, 2, BLOCK, h, d).transpose(0, 1)
        s["kcache"], s["vcache"] = pool[0], pool[1]
    table = torch.full((c["seqs"], max(blocks)), n_slots - 1, dtype=torch.int32, device=dev)
    slots = torch.randperm(n_slots, generator=gen, device=dev).int()
    at = 0
    for i, b in enumerate(blocks):
        table[i, :b] = slots[at:at + b]
        at += b
    start = np.concatenate([[0], np.cumsum(new)])
    s["table"] = table
    s["q_start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    s["max_new"], s["max_kv"], s["total"] = max(new), max(kv), int(start[-1])
    t = s["total"]
    if op in ("bounds", "select"):      # codes [slot, head, up / down, channel] and exponents [slot, head] of one layer
        if own:
            s["bounds"] = s["engine"].key_bounds(dt)
            s["codes"], s["exps"] = s["bounds"].codes[0], s["bounds"].exps[0]
        else:
            s["codes"] = torch.zeros(n_slots, h, 2, d, dtype=torch.int8, device=dev)
            s["exps"] = torch.zeros(n_slots, h, dtype=torch.uint8, device=dev)
    if op == "select":                  # as blocks of 16 normally distributed keys with a few strong channels leave them
        wide = torch.rand(h, 1, d, generator=gen, device=dev).pow(4).mul_(3).add_(0.3)
        reach = torch.randn(n_slots, h, 2, d, generator=gen, device=dev).mul_(0.5).add_(1.8).clamp_(0.2).mul_(wide)
        e = torch.ceil(torch.log2(reach.amax((2, 3)) / 127))
        s["codes"].copy_(torch.ceil(reach * torch.exp2(-e)[..., None, None]).clamp_(-127, 127))
        s["exps"].copy_(e + 127)
    if op in ("select", "sparse", "weigh"):
        # queries as a model's fused projection leaves them: slices of one row per token
        qkv = torch.empty(t, (g + 2) * h * d, dtype=dt, device=dev).normal_(generator=gen)
        s["q"] = qkv[:, :g * h * d].view(t, g * h, d).mul_(2.0)      # some keys matter and most do not, as in a trained model
    if op == "sparse":
        s["blocks"] = _some_blocks(s, gen)
    if op == "weigh":       # scores are distributed normally, with variance 4
        _, _, index = _where(s)
        seen = torch.clamp(index + 1, max=c["window"]) if c["window"] else index + 1
        s["lse"] = (seen.float().log() + 2.0)[:, None] + 0.2 * torch.randn(t, h * g, generator=gen, device=dev)
        s["weights"] = torch.rand(c["seqs"], max(blocks), generator=gen, device=dev).mul_(50.0)
    if op == "evict":       # a few blocks have most of the weight
        s["weights"] = torch.randn(c["seqs"], max(blocks), generator=gen, device=dev).mul_(2.0).exp_()
    return s


def _some_blocks(s, gen):
    """Lists as a selection leaves them: in order, the first and last blocks among them; neighbouring tokens choose alike."""
    c, dev = s["case"], "cuda"
    _, seq, index = _where(s)
    n, k = s["table"].shape[1], c["budget"]
    out = torch.empty(s["total"], c["kv_heads"], k, dtype=torch.int32, device=dev)
    for t0 in range(0, s["total"], 64):
        mine = (index[t0:t0 + 64] // BLOCK)[:, None, None]
        liking = torch.rand(1, c["kv_heads"], n, generator=gen, device=dev) + \
            0.5 * torch.rand(mine.shape[0], c["kv_heads"], n, generator=gen, device=dev)
        block = torch.arange(n, device=dev)
        liking = torch.where((block < c["first"]) | (block > mine - c["last"]), 2.0, liking).masked_fill(block > mine, -1.0)
        if n < k:
            liking = torch.nn.functional.pad(liking, (0, k - n), value=-1.0)
        best, which = liking.topk(k, -1)
        far = torch.iinfo(torch.int32).max
        which = which.int().masked_fill(best < 0, far).sort(-1).values
        out[t0:t0 + 64] = which.masked_fill(which == far, -1)
    return out


def _where(s):
    """Sequence and index in its sequence of every new token."""
    tok = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), tok, right=True)
    index = tok - s["q_start"].long()[seq + 1] + s["kv_len"].long()[seq]
    return tok, seq, index


def _power(e):
    """2^e in 64 bits, exactly, for whole numbers."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _steps(most, n):
    """Smallest e with most <= n * 2^e, where n is one less than a power of two."""
    m, e = torch.frexp(most / (n + 1))
    e = e - (m == 0.5).int()
    return torch.where(most.double() > n * _power(e), e + 1, e)


def _bounds(s):
    c = s["case"]
    _, seq, index = _where(s)
    last = index % BLOCK == BLOCK - 1       # the token fills its block
    slot = s["table"].long()[seq[last], index[last] // BLOCK]
    k = s["kcache"][slot].float()           # [block, token, head, channel]
    reach = torch.stack([k.amax(1), (-k).amax(1)], 2)
    most = k.abs().amax((1, 3))
    e = torch.where(most > 0, _steps(most, 127), -126)      # codes of at most 127 steps of 2^e
    s["codes"][slot] = torch.ceil(reach * _power(-e)[..., None, None]).to(torch.int8)
    s["exps"][slot] = (e + 127).to(torch.uint8)
    return {"codes": s["codes"], "exponents": s["exps"]}


def _query_codes(q, h, g):
    """The group's queries added up, above and below zero apart, in 8 bits without sign: rounded to steps of a power of two."""
    q = q.double().view(q.shape[0], h, g, -1)
    both = torch.stack([q.clamp(min=0).sum(2), (-q).clamp(min=0).sum(2)], 2)
    e = _steps(both.amax((2, 3)), 255)
    return torch.round(both * _power(-e)[..., None, None])      # [token, head, up / down, channel]


def _select(s):
    c = s["case"]
    h, g, k = c["kv_heads"], c["group"], c["budget"]
    _, seq, index = _where(s)
    t, n = s["total"], s["table"].shape[1]
    u = _query_codes(s["q"], h, g).float()
    table = s["table"].long()
    mine = index // BLOCK
    block = torch.arange(n, device="cuda")
    # sums of whole numbers below 2^24, times a power of two: nothing is rounded
    codes = s["codes"][table].float()
    value = _power(s["exps"][table].int() - 127).float()
    row = torch.arange(t, device="cuda") - s["q_start"].long()[seq]
    padded = torch.zeros(c["seqs"], s["max_new"], h, 2 * c["head_dim"], device="cuda")
    padded[seq, row] = u.flatten(2)
    score = padded.transpose(1, 2) @ codes.flatten(3).permute(0, 2, 3, 1) * value.permute(0, 2, 1)[:, :, None]
    score = score.transpose(1, 2)[seq, row]                 # [token, head, block]
    mine = mine[:, None, None]
    score = torch.where((block < c["first"]) | (block > mine - c["last"]), math.inf, score).masked_fill_(block > mine, -math.inf)
    order = score.argsort(dim=-1, descending=True, stable=True)[..., :k]
    order = torch.where(order <= mine, order, n).sort(-1).values.int()
    out = torch.full((t, h, k), -1, dtype=torch.int32, device="cuda")
    out[..., :order.shape[-1]] = order.masked_fill(order == n, -1)
    return {"blocks": out}


def _sparse(s):
    c = s["case"]
    h, g, d, k = c["kv_heads"], c["group"], c["head_dim"], c["budget"]
    _, seq, index = _where(s)
    t = s["total"]
    out = torch.empty(t, h * g, d, dtype=s["q"].dtype, device="cuda")
    lse = torch.empty(t, h * g, device="cuda")
    head = torch.arange(h, device="cuda")[:, None, None]
    step = max(1, 2 ** 30 // (h * k * BLOCK * d))           # tokens whose keys and values are gathered together
    for t0 in range(0, t, step):
        b = s["blocks"][t0:t0 + step].long()
        slot = s["table"].long()[seq[t0:t0 + step, None, None], b.clamp(min=0)]
        key = b[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")
        hidden = (b < 0)[..., None] | (key > index[t0:t0 + step, None, None, None])
        at = (slot[..., None], torch.arange(BLOCK, device="cuda"), head)
        kk = s["kcache"][at].float().flatten(2, 3)          # [token, head, key, channel]
        vv = s["vcache"][at].float().masked_fill(hidden[..., None], 0.0).flatten(2, 3)
        x = s["q"][t0:t0 + step].float().view(-1, h, g, d) @ kk.transpose(2, 3) * d ** -0.5
        x = x.masked_fill(hidden.flatten(2, 3)[:, :, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        x = (x - top).exp()
        total = x.sum(-1, keepdim=True)
        out[t0:t0 + step] = ((x @ vv) / total).flatten(1, 2).to(out.dtype)
        lse[t0:t0 + step] = (top + total.log()).flatten(1)
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def _weigh(s):
    c = s["case"]
    h, g, d = c["kv_heads"], c["group"], c["head_dim"]
    n, m, kv = c["seqs"], s["max_new"], s["max_kv"]
    tok, seq, index = _where(s)
    row = tok - s["q_start"].long()[seq]
    q = torch.zeros(n, m, h, g, d, device="cuda")
    q[seq, row] = s["q"].float().view(-1, h, g, d)
    lse = torch.zeros(n, m, h, g, device="cuda")
    lse[seq, row] = s["lse"].view(-1, h, g)
    own_index = torch.full((n, m), -1, dtype=torch.long, device="cuda")
    own_index[seq, row] = index
    k = s["kcache"][s["table"].long()].view(n, -1, h, d)[:, :kv].float()
    key = torch.arange(kv, device="cuda")
    hidden = key > own_index[..., None]
    if c["window"]:
        hidden |= key <= own_index[..., None] - c["window"]
    # [sequence, kv head, (query, group)] x [sequence, kv head, key]
    x = (q.permute(0, 2, 1, 3, 4).reshape(n, h, m * g, d) @ k.permute(0, 2, 3, 1)).mul_(d ** -0.5)
    x.sub_(lse.permute(0, 2, 1, 3).reshape(n, h, m * g, 1)).exp_()
    x.view(n, h, m, g, kv).masked_fill_(hidden[:, None, :, None], 0.0)
    per_key = x.sum((1, 2), dtype=torch.float64)
    blocks = s["table"].shape[1]
    per_block = torch.nn.functional.pad(per_key, (0, blocks * BLOCK - kv)).view(n, blocks, BLOCK).sum(-1)
    held = torch.arange(blocks, device="cuda") * BLOCK < s["kv_len"][:, None]
    return {"weights": (per_block + c["keep"] * s["weights"].double()).masked_fill(~held, 0.0).float()}


def _evict(s):
    c = s["case"]
    table, weights = s["table"], s["weights"]
    n = table.shape[1]
    had = (s["kv_len"] + BLOCK - 1) // BLOCK
    gone = (had - c["budget"]).clamp(min=0)
    block = torch.arange(n, device="cuda")
    mine = had[:, None]
    always = (block < c["first"]) | (block >= mine - c["last"])
    rank = torch.where(always, math.inf, weights).masked_fill(block >= mine, -math.inf)
    # place of every block among its sequence's by weight, the lower number first where weights are the same
    place = rank.argsort(dim=-1, descending=True, stable=True).argsort(dim=-1)
    kept = (place < c["budget"]) & (block < mine)

    def pack(x, which, empty):
        order = torch.where(which, block, n + block).sort(-1).indices
        return torch.where(block < which.sum(-1, keepdim=True), x.gather(-1, order), empty)

    return {"table": pack(table, kept, -1), "kv_len": s["kv_len"] - BLOCK * gone, "weights": pack(weights, kept, 0.0),
            "evicted": pack(table, ~kept & (block < mine), -1)}


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"bounds": _bounds, "select": _select, "sparse": _sparse, "weigh": _weigh, "evict": _evict}[c["op"]](s)
    eng = s["engine"]
    batch = (s["table"], s["q_start"], s["kv_len"])
    if c["op"] == "bounds":
        eng.bound_keys(0, s["bounds"], *batch, n_tokens=s["total"])
        return {"codes": s["codes"], "exponents": s["exps"]}
    if c["op"] == "select":
        return {"blocks": eng.select_blocks(0, s["q"], s["bounds"], *batch, c["budget"], first=c["first"], last=c["last"],
                                            max_q_len=s["max_new"])}
    if c["op"] == "sparse":
        lse = torch.empty(s["total"], c["kv_heads"] * c["group"], device="cuda") if c["lse"] else None
        o = eng.attend_blocks(0, s["q"], s["blocks"], *batch, lse=lse)
        return {"out": o, "lse": lse} if c["lse"] else {"out": o}
    if c["op"] == "weigh":
        return {"weights": eng.weigh_blocks(0, s["q"], s["lse"], *batch, max_q_len=s["max_new"], window=c["window"],
                                            weights=s["weights"], keep=c["keep"])}
    table, kv_len, weights, evicted = eng.evict_blocks(s["weights"], s["table"], s["kv_len"], c["budget"], first=c["first"],
                                                       last=c["last"])
    return {"table": table, "kv_len": kv_len, "weights": weights, "evicted": evicted}


def _exact_bounds(s, new, past):
    c = s["case"]
    codes, exps = s["codes"].clone(), s["exps"].clone()
    for i, (n, p) in enumerate(zip(new, past)):
        slot = s["table"][i, p // BLOCK:(p + n) // BLOCK].long()
        if not len(slot):
            continue
        k = s["kcache"][slot].double()
        most = k.abs().flatten(3).amax((1, 3))
        e = torch.full_like(most, -126.0)
        unit = torch.zeros_like(most)
        for p2 in range(20, -127, -1):       # the least power of two that holds the block's largest in 127 steps
            fits = most <= 127 * math.ldexp(1.0, p2)
            e, unit = e.masked_fill(fits, p2), unit.masked_fill(fits, math.ldexp(1.0, p2))
        unit = unit[:, :, None]
        codes[slot, :, 0] = torch.ceil(k.max(1).values / unit).to(torch.int8)
        codes[slot, :, 1] = (-torch.floor(k.min(1).values / unit)).to(torch.int8)
        exps[slot] = (e + 127).to(torch.uint8)
    return {"codes": codes, "exponents": exps}


def _exact_select(s, new, past):
    c = s["case"]
    h, g, d, k = c["kv_heads"], c["group"], c["head_dim"], c["budget"]
    out = torch.full((s["total"], h, k), -1, dtype=torch.int32, device="cuda")
    powers = torch.tensor([math.ldexp(1.0, e - 127) for e in range(256)], dtype=torch.float64, device="cuda")
    t0 = 0
    for i, (n, p) in enumerate(zip(new, past)):
        slots = s["table"][i, :(n + p - 1) // BLOCK + 1].long()
        mine = torch.arange(p, p + n, device="cuda") // BLOCK
        b = torch.arange(len(slots), device="cuda")
        for j in range(h):
            q = s["q"][t0:t0 + n, j * g:(j + 1) * g].double()
            up, down = torch.relu(q).sum(1), torch.relu(-q).sum(1)
            most = torch.maximum(up.max(1).values, down.max(1).values)
            unit = torch.zeros_like(most)
            for power in powers.flip(0):
                unit = torch.where(255 * power >= most, power, unit)
            unit = unit[:, None]
            above, below = (s["codes"][slots, j, y].double().T for y in (0, 1))
            x = torch.round(up / unit) @ above + torch.round(down / unit) @ below
            x = x * powers[s["exps"][slots, j].long()]
            x[(b < c["first"]) | (b > mine[:, None] - c["last"])] = math.inf
            x[b > mine[:, None]] = -math.inf
            best = torch.argsort(-x, dim=1, stable=True)[:, :k]
            chosen = torch.zeros_like(x, dtype=torch.bool).scatter_(1, best, True) & (b <= mine[:, None])
            at = chosen.cumsum(1) - 1
            r, col = chosen.nonzero(as_tuple=True)
            out[t0 + r, j, at[r, col]] = col.int()
        t0 += n
    return {"blocks": out}


def _exact_sparse(s, new, past):
    c = s["case"]
    h, g, d = c["kv_heads"], c["group"], c["head_dim"]
    out = torch.empty(s["total"], h * g, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["total"], h * g, dtype=torch.float64, device="cuda")
    t0 = 0
    for i, (n, p) in enumerate(zip(new, past)):
        slots = s["table"][i, :(n + p - 1) // BLOCK + 1].long()
        own_index = torch.arange(p, p + n, device="cuda")[:, None]
        for j in range(h):
            k = s["kcache"][slots, :, j].double().flatten(0, 1)
            v = s["vcache"][slots, :, j].double().flatten(0, 1)
            chosen = torch.zeros(n, len(slots) + 1, dtype=torch.bool, device="cuda")
            mine = s["blocks"][t0:t0 + n, j].long()
            chosen.scatter_(1, torch.where(mine < 0, len(slots), mine), True)
            see = chosen[:, :-1].repeat_interleave(BLOCK, 1) & (torch.arange(len(k), device="cuda") <= own_index)
            for r in range(j * g, j * g + g):
                x = torch.where(see, (s["q"][t0:t0 + n, r].double() @ k.T) / math.sqrt(d), -math.inf)
                lse[t0:t0 + n, r] = torch.logsumexp(x, 1)
                out[t0:t0 + n, r] = torch.exp(x - lse[t0:t0 + n, r:r + 1]) @ v
        t0 += n
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def _exact_weigh(s, new, past):
    c = s["case"]
    h, g, d = c["kv_heads"], c["group"], c["head_dim"]
    out = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda")
    t0 = 0
    for i, (n, p) in enumerate(zip(new, past)):
        blocks = -(-(n + p) // BLOCK)
        slots = s["table"][i, :blocks].long()
        own_index = torch.arange(p, p + n, device="cuda")[:, None]
        key = torch.arange(blocks * BLOCK, device="cuda")
        see = key <= own_index
        if c["window"]:
            see &= own_index - key < c["window"]
        total = torch.zeros(blocks * BLOCK, dtype=torch.float64, device="cuda")
        for j in range(h):
            k = s["kcache"][slots, :, j].double().flatten(0, 1)
            for r in range(j * g, j * g + g):
                x = s["q"][t0:t0 + n, r].double() @ k.T / math.sqrt(d) - s["lse"][t0:t0 + n, r:r + 1].double()
                total += torch.where(see, x.exp(), 0.0).sum(0)
        out[i, :blocks] = c["keep"] * s["weights"][i, :blocks].double() + total.view(-1, BLOCK).sum(1)
        t0 += n
    return {"weights": out}


def _exact_evict(s, new, past):
    c = s["case"]
    table, weights = s["table"].cpu().numpy(), s["weights"].cpu().numpy()
    got = {"table": np.full_like(table, -1), "kv_len": np.zeros(len(table), np.int32), "weights": np.zeros(weights.shape),
           "evicted": np.full_like(table, -1)}
    for i, (n, p) in enumerate(zip(new, past)):
        had = -(-(n + p) // BLOCK)
        free = list(range(c["first"], max(c["first"], had - c["last"])))
        free.sort(key=lambda b: (weights[i, b], -b))        # least weight first, of the same the higher number
        gone = sorted(free[:max(0, had - c["budget"])])
        kept = np.setdiff1d(np.arange(had), gone)
        got["table"][i, :len(kept)], got["weights"][i, :len(kept)] = table[i, kept], weights[i, kept]
        got["evicted"][i, :len(gone)] = table[i, gone]
        got["kv_len"][i] = n + p - BLOCK * len(gone)
    return {k: torch.from_numpy(v) for k, v in got.items()}


def exact(case, seed):
    """The definitions, sequence by sequence and head by head, in 64 bits or in whole numbers."""
    s = prepare(case, seed)
    return {"bounds": _exact_bounds, "select": _exact_select, "sparse": _exact_sparse, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["op"]](s, *_lengths(case))
