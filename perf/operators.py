"""The model-side operators on the engine's KV pool, as a serving loop uses them, with the sizes they are measured at.

append: the new tokens' keys and values are rotated by their positions and written into the pool's blocks, and the
        queries are rotated with them.
attend: the queries of a chunk of new tokens (or of one new token per sequence) attend to everything their sequence
        has in the pool.

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
    c = dict(op=op, dtype="bf16", layout=0, layers=2, layer=1, kv_heads=8, group=4, head_dim=128, seqs=1, new_lo=1,
             new_hi=1, past_lo=0, past_hi=0, mix=1)
    c.update(dict(axes=1, rot=128, interleaved=False, theta=10000.0) if op == "append" else dict(window=0, lse=False))
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one decode step of 32 sessions, 8B-class heads: all launch latency
        _case("append", "append step 32", seqs=32, past_lo=100, past_hi=8000),
        # prefill of one 8 K prompt, 8B-class heads
        _case("append", "append prompt 8k", new_lo=8192, new_hi=8192, theta=500000.0),
        # images and video: three position axes, fp16, small heads, block-major pool, odd lengths
        _case("append", "append axes ragged", dtype="fp16", layout=1, kv_heads=2, group=7, head_dim=64, rot=64, seqs=9,
              new_lo=33, new_hi=1500, past_lo=0, past_hi=900, axes=3, mix=5),
        # agent contexts that bring long tool results far into their sequences, half of each head rotated
        _case("append", "append batch 64k", seqs=9, group=12, new_lo=2000, new_hi=14000, past_lo=6000, past_hi=90000,
              layers=1, layer=0, rot=64, interleaved=True, mix=3),
        # one new token of one short session: latency
        _case("attend", "step 1 x 1k", past_lo=1000, past_hi=1000),
        # one new token of one long agent session (258 K tokens)
        _case("attend", "step 1 x 258k", past_lo=258047, past_hi=258047, layers=1, layer=0),
        # one new token each of 32 sessions of very different lengths, wide groups
        _case("attend", "step 32 ragged", seqs=32, group=12, past_lo=2000, past_hi=130000, layers=1, layer=0, mix=2,
              lse=True),
        # many short sessions, small heads without grouping, fp16, block-major
        _case("attend", "step 96 toy", dtype="fp16", layout=1, kv_heads=2, group=1, head_dim=64, seqs=96, past_lo=1,
              past_hi=3000, mix=7),
        # prefill of one 8 K prompt
        _case("attend", "prompt 8k", new_lo=8192, new_hi=8192),
        # a chunk of new tokens (a tool result) at the end of a long session
        _case("attend", "chunk 500 x 128k", new_lo=500, new_hi=500, past_lo=130500, past_hi=130500, layers=1, layer=0,
              lse=True),
        # several sessions bring tool results of odd lengths, small heads, fp16, sliding window, block-major
        _case("attend", "ragged window 1k", dtype="fp16", layout=1, kv_heads=4, group=8, head_dim=64, seqs=7, new_lo=65,
              new_hi=1300, past_lo=0, past_hi=7000, window=1024, mix=4),
        # decoding sessions and sessions in prefill in the same batch
        _case("attend", "mixed batch", seqs=8, new_lo=1, new_hi=700, past_lo=16, past_hi=16000, mix=6),
    ]


def _between(rng, lo, hi):
    """Whole number in [lo, hi], spread over its logarithm."""
    return min(hi, int((lo + 1) * math.exp(rng.random() * math.log((hi + 1.999) / (lo + 1)))) - 1)


def draw(rng):
    """A case of the same ranges: whichever operator, 1 .. 64 sequences, prompts from one token up."""
    heads, head_dim = rng.choice([(2, 64), (4, 64), (4, 128), (8, 128), (1, 128)])
    c = dict(dtype=rng.choice(["bf16", "fp16"]), layout=rng.randrange(2), kv_heads=heads, head_dim=head_dim, layers=1,
             layer=0, group=rng.choice([1, 2, 3, 4, 7, 8, 12]), mix=rng.randrange(1 << 20))
    if rng.random() < 0.35:
        total = _between(rng, 1, 40000)
        seqs = _between(rng, 1, min(total, 64))
        new = -(-total // seqs)
        rot = rng.choice([head_dim, head_dim // 2])
        return _case("append", seqs=seqs, new_lo=_between(rng, 1, new), new_hi=new, past_hi=_between(rng, 0, 100000 // seqs),
                     axes=rng.choice([1, 1, 3]), rot=rot, interleaved=rng.random() < 0.5,
                     theta=rng.choice([10000.0, 500000.0]), **c)
    window = rng.choice([0, 0, 0, _between(rng, 16, 4096)])
    lse = rng.random() < 0.5
    if rng.random() < 0.5:      # decode
        total = _between(rng, 1000, 1400000)
        seqs = _between(rng, 1, 64)
        hi = min(250000, total // seqs + 1)
        return _case("attend", seqs=seqs, past_lo=_between(rng, 0, hi), past_hi=hi, window=window, lse=lse, **c)
    total = _between(rng, 10, 6000)      # prompts and chunks
    seqs = _between(rng, 1, 8)
    new = total // seqs + 1
    past = _between(rng, 0, 30000000 // (total + 500) // seqs)
    return _case("attend", seqs=seqs, new_lo=_between(rng, 1, new), new_hi=new, past_lo=0, past_hi=past, window=window,
                 lse=lse, **c)


def _lengths(case):
    """New and cached tokens of every sequence; they belong to the case, not to the seed."""
    rng = random.Random(case["mix"])
    pick = lambda lo, hi: _between(rng, min(lo, hi), hi)  # noqa: E731
    return ([pick(case["new_lo"], case["new_hi"]) for _ in range(case["seqs"])],
            [pick(case["past_lo"], case["past_hi"]) for _ in range(case["seqs"])])


def _seen(case):
    """Number of (query, key) pairs that the mask leaves, over all sequences, and of keys that any query sees."""
    pairs = keys = 0
    for n, p in zip(*_lengths(case)):
        w = case["window"] or n + p
        i = np.arange(p + 1, p + n + 1, dtype=np.int64)      # keys up to and with each query's own
        pairs += int(np.minimum(i, w).sum())
        keys += min(n + p, w + n - 1)
    return pairs, keys


def work(case):
    h, d, g = case["kv_heads"], case["head_dim"], case["group"]
    t = sum(_lengths(case)[0])
    if case["op"] == "append":      # q, k, v read once and written once
        return {"bytes": 2 * 2 * t * h * d * (g + 2), "flops": 3 * t * h * case["rot"] * (g + 1)}
    pairs, keys = _seen(case)
    return {"bytes": 2 * (2 * keys * h * d + 2 * t * h * g * d) + (4 * t * h * g if case["lse"] else 0),
            "flops": 4 * pairs * h * g * d}


def prepare(case, seed):
    c, dev = case, "cuda"
    gen = torch.Generator(dev).manual_seed(seed * 1000003 + 17)
    dt = DTYPES[c["dtype"]]
    new, past = _lengths(c)
    kv = [n + p for n, p in zip(new, past)]
    blocks = [-(-n // BLOCK) for n in kv]
    n_slots = sum(blocks) + 3 + sum(blocks) // 50
    chunks, h, d = 2 * c["layers"], c["kv_heads"], c["head_dim"]
    s = {"case": c}
    if own:
        from paper_2609_39819_b200 import binding
        s["engine"] = binding.Engine(n_layers=c["layers"], n_kv_heads=h, head_dim=d, pool_layout=c["layout"],
                                     n_hbm_blocks=n_slots, n_host_blocks=0, max_contexts=1, max_messages=16,
                                     max_tokens=64, zero_pools=False)
        pool = s["engine"].hbm_pool.view(dt)
    else:
        pool = torch.empty(chunks * n_slots * BLOCK * h * d, dtype=dt, device=dev)
    pool.normal_(generator=gen)
    # one layer's K and V as [slot, token, head, dim]
    pool = pool.view(chunks, n_slots, BLOCK, h, d) if c["layout"] == 0 else \
        pool.view(n_slots, chunks, BLOCK, h, d).transpose(0, 1)
    s["pool"], s["kcache"], s["vcache"] = pool, pool[2 * c["layer"]], pool[2 * c["layer"] + 1]
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
    # q, k and v as a model's fused projection leaves them: slices of one row per token
    qkv = torch.empty(t, (c["group"] + 2) * h * d, dtype=dt, device=dev).normal_(generator=gen)
    s["q"] = qkv[:, :c["group"] * h * d].view(t, c["group"] * h, d)
    if c["op"] == "append":
        s["k"] = qkv[:, c["group"] * h * d:-h * d].view(t, h, d)
        s["v"] = qkv[:, -h * d:].view(t, h, d)
        pairs = c["rot"] // 2
        sections = [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8] if c["axes"] == 3 else [pairs]
        s["axis_of"] = torch.repeat_interleave(torch.arange(c["axes"], device=dev), torch.tensor(sections, device=dev))
        s["positions"] = None
        if c["axes"] == 3:   # time runs on, height and width lie on a grid
            s["positions"] = torch.stack([torch.arange(t, device=dev) // 7 + past[0],
                                          torch.randint(0, 64, (t,), generator=gen, device=dev),
                                          torch.randint(0, 96, (t,), generator=gen, device=dev)]).int()
        if own:
            s["rope"] = binding.Rope(c["rot"], theta=c["theta"], sections=sections if c["axes"] == 3 else None,
                                     interleaved=c["interleaved"])
    else:
        s["q"].mul_(2.0)     # some keys matter and most do not, as in a trained model
    return s


def _where(s):
    """Sequence and index in its sequence of every new token."""
    tok = torch.arange(s["total"], device="cuda")
    seq = torch.searchsorted(s["q_start"][1:].long(), tok, right=True)
    index = tok - s["q_start"].long()[seq + 1] + s["kv_len"].long()[seq]
    return tok, seq, index


def _rotate(x, cos, sin, interleaved):
    """x: [tokens, heads, rot] in 32 bits; cos, sin: [tokens, rot / 2]."""
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
    else:
        a, b = x.chunk(2, -1)
    a, b = a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]
    return torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)


def _append(s):
    c = s["case"]
    _, seq, index = _where(s)
    rot, dt = c["rot"], s["q"].dtype
    freq = c["theta"] ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    pos = index[None] if s["positions"] is None else s["positions"]
    angle = pos.double().T[:, s["axis_of"]] * freq          # 64 bits: far positions turn many times
    cos, sin = angle.cos().float(), angle.sin().float()

    def turned(x):
        return torch.cat([_rotate(x[..., :rot].float(), cos, sin, c["interleaved"]), x[..., rot:].float()], -1).to(dt)

    slot = s["table"].long()[seq, index // BLOCK]
    s["kcache"][slot, index % BLOCK] = turned(s["k"])
    s["vcache"][slot, index % BLOCK] = s["v"]
    return {"q": turned(s["q"]), "pool": s["pool"]}


def _attend(s):
    c = s["case"]
    h, g, d = c["kv_heads"], c["group"], c["head_dim"]
    n, m, kv = c["seqs"], s["max_new"], s["max_kv"]
    tok, seq, index = _where(s)
    row = tok - s["q_start"].long()[seq]
    q = torch.zeros(n, m, h, g, d, device="cuda")
    q[seq, row] = s["q"].float().view(-1, h, g, d)
    own_index = torch.zeros(n, m, dtype=torch.long, device="cuda")
    own_index[seq, row] = index
    table = s["table"].long()[:, :-(-kv // BLOCK)]
    k = s["kcache"][table].view(n, -1, h, d)[:, :kv].float()
    v = s["vcache"][table].view(n, -1, h, d)[:, :kv].float()
    key = torch.arange(kv, device="cuda")
    hidden = key > own_index[..., None]
    if c["window"]:
        hidden |= key <= own_index[..., None] - c["window"]
    v = v.masked_fill((key >= s["kv_len"][:, None])[..., None, None], 0.0)
    # [sequence, kv head, (query, group)] x [sequence, kv head, key]
    x = (q.permute(0, 2, 1, 3, 4).reshape(n, h, m * g, d) @ k.permute(0, 2, 3, 1)) * d ** -0.5
    x.view(n, h, m, g, kv).masked_fill_(hidden[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ v.permute(0, 2, 1, 3)) / total
    o = o.view(n, h, m, g, d).permute(0, 2, 1, 3, 4)[seq, row].reshape(-1, h * g, d).to(s["q"].dtype)
    if not c["lse"]:
        return {"out": o}
    lse = (top + total.log()).view(n, h, m, g).permute(0, 2, 1, 3)[seq, row].reshape(-1, h * g)
    return {"out": o, "lse": lse}


def run(state):
    s, c = state, state["case"]
    if not own:
        return _append(s) if c["op"] == "append" else _attend(s)
    eng = s["engine"]
    if c["op"] == "append":
        q = eng.append_kv(c["layer"], s["k"], s["v"], s["table"], s["q_start"], s["kv_len"], rope=s["rope"],
                          positions=s["positions"], q=s["q"])
        return {"q": q, "pool": s["pool"]}
    lse = torch.empty(s["total"], c["kv_heads"] * c["group"], device="cuda") if c["lse"] else None
    o = eng.attend(c["layer"], s["q"], s["table"], s["q_start"], s["kv_len"], max_q_len=s["max_new"],
                   window=c["window"], lse=lse)
    return {"out": o, "lse": lse} if c["lse"] else {"out": o}


def exact(case, seed):
    """The definitions, sequence by sequence and head by head, in 64 bits."""
    c = case
    s = prepare(case, seed)
    new, past = _lengths(c)
    h, g, d = c["kv_heads"], c["group"], c["head_dim"]
    out_q, out_lse, t0 = [], [], 0
    if c["op"] == "append":
        pool = s["pool"].double()
    for i, (n, p) in enumerate(zip(new, past)):
        q = s["q"][t0:t0 + n].double()
        rows = s["table"][i].long().repeat_interleave(BLOCK) * BLOCK + \
            torch.arange(BLOCK, device="cuda").repeat(s["table"].shape[1])
        if c["op"] == "append":
            at = torch.arange(p, p + n, device="cuda")
            axis = [int(a) for a in s["axis_of"].cpu()]
            x = torch.cat([q, s["k"][t0:t0 + n].double()], 1)
            y = x.clone()
            for j in range(c["rot"] // 2):
                where = at if s["positions"] is None else s["positions"][axis[j], t0:t0 + n]
                a = where.double() * math.pow(c["theta"], -2.0 * j / c["rot"])
                u, w = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + c["rot"] // 2)
                z = torch.polar(torch.ones_like(a), a)[:, None] * torch.complex(x[..., u], x[..., w])
                y[..., u], y[..., w] = z.real, z.imag
            out_q.append(y[:, :h * g])
            slot, off = rows[p:p + n] // BLOCK, rows[p:p + n] % BLOCK
            pool[2 * c["layer"], slot, off] = y[:, h * g:]
            pool[2 * c["layer"] + 1, slot, off] = s["v"][t0:t0 + n].double()
        else:
            rows = rows[:p + n]
            o = torch.empty(n, h * g, d, dtype=torch.float64, device="cuda")
            lse = torch.empty(n, h * g, dtype=torch.float64, device="cuda")
            mine, key = torch.arange(p, p + n, device="cuda")[:, None], torch.arange(p + n, device="cuda")[None]
            see = key <= mine
            if c["window"]:
                see &= mine - key < c["window"]
            for j in range(h):
                k = s["kcache"][rows // BLOCK, rows % BLOCK, j].double()
                v = s["vcache"][rows // BLOCK, rows % BLOCK, j].double()
                for r in range(j * g, j * g + g):
                    x = (q[:, r] @ k.T) / math.sqrt(d)
                    x = torch.where(see, x, -math.inf)
                    lse[:, r] = torch.logsumexp(x, 1)
                    o[:, r] = torch.exp(x - lse[:, r:r + 1]) @ v
            out_q.append(o)
            out_lse.append(lse)
        t0 += n
    if c["op"] == "append":
        return {"q": torch.cat(out_q), "pool": pool}
    return {"out": torch.cat(out_q), "lse": torch.cat(out_lse)} if c["lse"] else {"out": torch.cat(out_q)}
