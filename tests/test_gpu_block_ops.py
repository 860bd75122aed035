"""bound_keys, select_blocks, attend_blocks, weigh_blocks and evict_blocks against their definitions in 64 bits or in whole numbers.
Unused parts of the pool hold NaN, so anything read that should not be shows up."""
import ctypes as C
import math

import numpy as np
import pytest

from test_gpu_model_ops import B, BT, Setup, rotated  # noqa: F401

pytestmark = pytest.mark.gpu
E32 = 2.0 ** -24


# ---- definitions --------------------------------------------------------------------------------
def bounds_of(torch, k):
    """k: [16, heads, dim] in 64 bits. Codes [heads, 2, dim] and exponents [heads]."""
    top = 3.3895313892515355e38
    k = torch.where(torch.isnan(k), torch.nan, k)
    hi = torch.where(torch.isnan(k), -math.inf, k).amax(0)
    lo = torch.where(torch.isnan(k), math.inf, k).amin(0)
    none = torch.isnan(k).all(0)
    hi, lo = hi.masked_fill(none, 0.0).clamp(-4 * top, 4 * top), lo.masked_fill(none, 0.0).clamp(-4 * top, 4 * top)
    most = torch.maximum(hi.abs(), lo.abs()).amax(-1)
    exps = torch.tensor([next((e for e in range(-126, 103) if m <= 127 * math.ldexp(1.0, e)), 103) for m in most.tolist()])
    unit = torch.tensor([math.ldexp(1.0, int(e)) for e in exps], dtype=torch.float64, device=k.device)[:, None]
    codes = torch.stack([torch.ceil(hi / unit), torch.ceil(-lo / unit)], 1).clamp(-127, 127)
    return codes.to(torch.int8), exps


def lists_of(torch, q, codes, exps, index, group, n_blocks, first, last):
    """q: [tokens, heads, dim] of one sequence; codes [blocks, KV heads, 2, dim], exps [blocks, KV heads] (e + 127) of its blocks in
    order; index: of the tokens. The lists, [tokens, KV heads, n_blocks]."""
    heads = q.shape[1] // group
    top = torch.finfo(q.dtype).max
    q = torch.nan_to_num(q.double(), nan=0.0, posinf=top, neginf=-top)
    q = q.view(len(q), heads, group, q.shape[-1])
    both = torch.stack([q.clamp(min=0).sum(2), (-q).clamp(min=0).sum(2)], 2).cpu().numpy()
    codes, exps = codes.cpu().numpy().astype(np.int64), exps.cpu().numpy().astype(int)
    d = both.shape[-1]
    out = np.full((len(index), heads, n_blocks), -1, np.int32)
    for t, i in enumerate(index):
        own = i // BT
        for h in range(heads):
            if own < n_blocks:
                out[t, h, :max(0, own + 1)] = np.arange(max(0, own + 1))
                continue
            most = both[t, h].max()
            f = next((f for f in range(-160, 160) if most <= 255 * math.ldexp(1.0, f)), 0) if most > 0 else 0
            u = np.rint(both[t, h] * math.ldexp(1.0, -f)).astype(np.int64)
            free = range(first, own + 1 - last)
            s = (codes[free.start:free.stop, h, :, :d] * u).sum((1, 2)).astype(np.float64)
            e = exps[free.start:free.stop, h]
            s *= np.where(e > 0, np.ldexp(1.0, e - 127), 0.0)
            best = np.argsort(-s, kind="stable")[:n_blocks - first - last] + first
            out[t, h] = np.concatenate([np.arange(first), np.sort(best), np.arange(own + 1 - last, own + 1)])
    return out


def sparse_reference(s, blocks, scale=None):
    """out, lse and how far each may be off. blocks: [tokens, KV heads, n]."""
    torch = s.torch
    scale = s.dim ** -0.5 if scale is None else scale
    hq = s.heads * s.group
    out = torch.zeros(s.t, hq, s.dim, dtype=torch.float64, device="cuda")
    lse = torch.full((s.t, hq), -math.inf, dtype=torch.float64, device="cuda")
    tol, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    t0 = 0
    for i, n in enumerate(s.new):
        k, v = s.gather(i)
        for t in range(n):
            index = s.kv[i] - n + t
            for kh in range(s.heads):
                listed = [b for b in blocks[t0 + t, kh].tolist() if b >= 0]
                keys = [j for b in listed for j in range(b * BT, min(b * BT + BT, index + 1))]
                if not keys:
                    continue
                kk, vv = k[keys, kh], v[keys, kh]
                hs = slice(kh * s.group, (kh + 1) * s.group)
                q = s.q[t0 + t, hs].double()
                x = q @ kk.T * scale
                big = (q.abs() @ kk.abs().T * abs(scale)).amax(1, keepdim=True)
                L = torch.logsumexp(x, 1, keepdim=True)
                p = torch.exp(x - L)
                o = p @ vv
                out[t0 + t, hs], lse[t0 + t, hs] = o, L[:, 0]
                # scores: dim products summed in 32 bits and the scaling; sums over the keys in 32 bits; powers as two numbers of the
                # element type, which leaves u^2 of each (fp16: or its fixed step); the result rounded once
                ds, sums = (s.dim + 4) * E32 * big, (len(keys) + 64) * E32
                tol[t0 + t, hs] = s.u * o.abs() + p @ vv.abs() * (s.u ** 2 + 2 * ds + 2 * sums) * (1 + s.u)
                if s.dt == torch.float16:
                    tol[t0 + t, hs] += 2.0 ** -25 * (1 + vv.abs().sum(0) * torch.exp(x.amax(1, keepdim=True) - L))
                tol_l[t0 + t, hs] = (ds + sums)[:, 0] + 4 * E32 * L[:, 0].abs()
        t0 += n
    return out, lse, tol, tol_l


def weights_reference(s, lse, window=0, causal=True, scale=None):
    """New weights per block [sequences, blocks of a row] and how far each may be off."""
    torch = s.torch
    scale = s.dim ** -0.5 if scale is None else float(np.float32(scale))
    width = s.table.shape[1]
    out = torch.zeros(len(s.new), width * BT, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    t0 = 0
    for i, n in enumerate(s.new):
        k, _ = s.gather(i)
        kv = s.kv[i]
        own = torch.arange(n, device="cuda")[:, None] + (kv - n)
        key = torch.arange(kv, device="cuda")[None]
        see = (key <= own) if causal else torch.ones(n, kv, dtype=torch.bool, device="cuda")
        if window:
            see &= own - key < window
        for h in range(s.heads * s.group):
            if not n or not kv:
                continue
            q, kh = s.q[t0:t0 + n, h].double(), k[:, h // s.group]
            L = lse[t0:t0 + n, h:h + 1].double()
            x = q @ kh.T * scale
            p = torch.where(see & torch.isfinite(L), torch.exp(x - L), 0.0)
            # the score: dim products summed in 32 bits; its difference to lse: three roundings of numbers up to |x| + |lse|; the
            # power: 2^-22; all relative to the power
            d = (s.dim + 2) * E32 * (q.abs() @ kh.abs().T) * abs(scale) + 4 * E32 * (x.abs() + L.abs()) + 2.0 ** -22
            out[i, :kv] += p.sum(0)
            tol[i, :kv] += torch.where(p > 0, p * torch.expm1(torch.where(p > 0, d, 0.0)), 0.0).sum(0)
        t0 += n
    per_block = lambda x: x.view(len(s.new), width, BT).sum(-1)      # noqa: E731
    out, tol = per_block(out), per_block(tol)
    rows = max(s.new + [1]) * s.heads * s.group * BT
    # sums in 32 bits, whatever their order; powers below 2^-126, the least number of 32 bits, may count as 0
    return out, tol + out * E32 * (rows + 8) + rows * 2.0 ** -126


BATCHES = {
    "step": ([1, 1, 1], [0, 15, 200]),
    "fills": ([1, 16, 3, 40], [15, 0, 30, 700]),
    "ragged": ([5, 0, 33, 1], [300, 20, 90, 3]),
    "prompt": ([70], [0]),
    "empty": ([0, 2, 0], [0, 500, 10]),
}
HEADS = [("bf16", 0, 2, 4, 128), ("fp16", 1, 2, 1, 64), ("bf16", 1, 1, 7, 64), ("fp16", 0, 3, 12, 128), ("bf16", 0, 2, 3, 16),
         ("fp16", 1, 8, 2, 40), ("bf16", 0, 1, 17, 72), ("bf16", 1, 2, 2, 256), ("fp16", 0, 1, 3, 7)]


def make(B, batch, dtype, layout, heads, group, dim, **kw):  # noqa: F811
    new, past = BATCHES[batch] if isinstance(batch, str) else batch
    s = Setup(B, new, past, heads, group, dim, dtype, layout, **kw)
    s.put()
    return s


# ---- bounds -------------------------------------------------------------------------------------
def check_bounds(s, n_tokens=None):
    torch = s.torch
    k = s.eng.key_bounds(s.dt)
    k.codes.fill_(77)
    k.exps.fill_(78)
    want_c, want_e = k.codes.clone(), k.exps.clone()
    s.eng.bound_keys(s.layer, k, s.table, s.q_start, s.kv_len, n_tokens=s.rows if n_tokens is None else n_tokens)
    s.eng.kv_check()
    for i, (n, kv) in enumerate(zip(s.new, s.kv)):
        for b in range((kv - n) // BT, kv // BT):
            slot = int(s.host_table[i, b])
            c, e = bounds_of(torch, s._chunk(slot, 0).double())
            want_c[s.layer, slot] = 0
            want_c[s.layer, slot, :, :, :s.dim] = c
            want_e[s.layer, slot] = (e + 127).to(torch.uint8).cuda()
    assert torch.equal(k.codes, want_c) and torch.equal(k.exps, want_e)


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("dtype,layout,heads,group,dim", HEADS)
def test_bounds(B, batch, dtype, layout, heads, group, dim):  # noqa: F811
    check_bounds(make(B, batch, dtype, layout, heads, group, dim, tail=batch != "step", pad=3))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 24])
def test_bounds_of_strange_keys(B, dtype, dim):  # noqa: F811
    """Zeros, NaN, Inf, the largest and the smallest numbers, and numbers next to 127 steps of a power of two."""
    import torch
    s = make(B, ([160], [0]), dtype, 0, 1, 1, dim)
    f = torch.finfo(s.dt)
    k = [s._chunk(int(x), 0)[:, 0] for x in s.host_table[0, :10]]
    k[0].zero_()
    k[1].fill_(math.nan)
    k[2][3].fill_(math.nan)
    k[3][5, 7] = math.inf
    k[4][:, 2] = -math.inf
    k[5].mul_(f.tiny).mul_(f.eps)
    k[6].mul_(f.tiny)
    k[6][1, 1] = f.max
    k[7].clamp_(-1, 1)
    k[7][2, 2] = 127 / 64
    k[8].clamp_(-1, 1)
    k[8][2, 2] = -127.5 / 64
    k[9].clamp_(max=-0.25)
    check_bounds(s)


def test_bounds_by_a_batch_that_counts_cached_tokens_as_new(B):  # noqa: F811
    s = make(B, ([300, 7, 64], [0, 0, 0]), "bf16", 0, 2, 1, 128)
    check_bounds(s)
    s.new = [300, 7, 64]
    check_bounds(s, n_tokens=371)


# ---- selection ----------------------------------------------------------------------------------
def random_bounds(s, g, span=6):
    """Bounds of every slot, with exponents `span` apart."""
    torch = s.torch
    k = s.eng.key_bounds(s.dt)
    k.codes.random_(-127, 128, generator=g)
    k.codes[..., s.dim:] = 0
    k.exps.random_(120, 120 + span, generator=g)
    return k


def check_select(s, k, n_blocks, first, last, table=None, **kw):
    torch = s.torch
    table = s.table if table is None else table
    out = torch.full((s.rows, s.heads, n_blocks), -7, dtype=torch.int32, device="cuda")
    got = s.eng.select_blocks(s.layer, s.q, k, table, s.q_start, s.kv_len, n_blocks, first=first, last=last, out=out, **kw)
    assert got is out
    s.eng.kv_check()
    t0 = 0
    for i, n in enumerate(s.new):
        slots = s.host_table[i, :-(-s.kv[i] // BT)].long().cuda()
        want = lists_of(torch, s.q[t0:t0 + n], k.codes[s.layer, slots], k.exps[s.layer, slots], [s.kv[i] - n + t for t in range(n)],
                        s.group, n_blocks, first, last)
        assert np.array_equal(out[t0:t0 + n].cpu().numpy(), want)
        t0 += n
    assert bool((out[s.t:] == -7).all())


@pytest.mark.parametrize("n_blocks,first,last", [(8, 1, 2), (3, 0, 1), (5, 2, 3), (1, 0, 1), (40, 1, 2)])
@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("dtype,layout,heads,group,dim", HEADS)
def test_select(B, batch, dtype, layout, heads, group, dim, n_blocks, first, last):  # noqa: F811
    import torch
    s = make(B, batch, dtype, layout, heads, group, dim, tail=True, pad=2, strided=heads == 2)
    check_select(s, random_bounds(s, torch.Generator("cuda").manual_seed(dim)), n_blocks, first, last)


@pytest.mark.parametrize("n_blocks,first,last", [(60, 21, 17), (40, 9, 31), (90, 0, 1), (64, 63, 1)])
def test_select_many_first_and_last(B, n_blocks, first, last):  # noqa: F811
    import torch
    s = make(B, ([5, 1], [1500, 7000]), "bf16", 0, 2, 2, 64)
    check_select(s, random_bounds(s, torch.Generator("cuda").manual_seed(8)), n_blocks, first, last)


def test_select_in_parts(B):  # noqa: F811
    """More scores than are in hand together, since the table could hold many more blocks: parts that end inside a sequence."""
    import torch
    s = make(B, ([700, 600], [900, 3000]), "fp16", 0, 2, 2, 16, pad=3)
    k = random_bounds(s, torch.Generator("cuda").manual_seed(8))
    wide = torch.full((2, 20000), -1, dtype=torch.int32, device="cuda")
    wide[:, :s.table.shape[1]] = s.table
    want = s.eng.select_blocks(1, s.q, k, s.table, s.q_start, s.kv_len, 30)
    got = s.eng.select_blocks(1, s.q, k, wide, s.q_start, s.kv_len, 30)
    s.eng.kv_check()
    assert torch.equal(want[:s.t], got[:s.t])
    t0 = 0
    for i, n in enumerate(s.new):
        slots = s.host_table[i, :-(-s.kv[i] // BT)].long().cuda()
        some = list(range(0, n, 37))
        ref = lists_of(torch, s.q[[t0 + x for x in some]], k.codes[1, slots], k.exps[1, slots], [s.kv[i] - n + x for x in some], 2, 30, 1, 2)
        assert np.array_equal(got[[t0 + x for x in some]].cpu().numpy(), ref)
        t0 += n


@pytest.mark.parametrize("n_tokens,width,heads", [(1, 100, 8), (500, 8157, 8), (600, 8157, 8), (700, 8157, 8), (5000, 4063, 8), (33, 1 << 20, 1), (3, 1 << 22, 8), (90000, 700, 2)])
def test_select_parts_are_alike(B, n_tokens, width, heads):  # noqa: F811
    """The scratch is that of parts of equal length (up to 31 tokens apart), no more of them than 128 MiB of scores each make necessary."""
    import torch
    eng = B.Engine(n_layers=1, n_kv_heads=heads, head_dim=16, n_hbm_blocks=4, n_host_blocks=0, max_contexts=1, max_messages=16, max_tokens=64)
    k = eng.key_bounds(torch.bfloat16)
    a = B.SelectArgs(B.Batch(1, n_tokens, width, 0, width, 16, 16, 16), 0, 0, heads, 9, 1, 2, 0, heads * 16, 16, eng._bounds("", k), 0, 0, 0)
    got = eng.L.kvt_select_scratch_bytes(eng.h, C.byref(a))
    token = (width + 7) // 8 * 8 * heads * 4
    most = max(1, (128 << 20) // token)
    parts = -(-n_tokens // most)
    assert got % token == 0 and -(-n_tokens // parts) <= got // token <= min(most, -(-n_tokens // parts) + 31)


@pytest.mark.parametrize("span", [1, 3])
@pytest.mark.parametrize("codes", [1, 2, 127])
def test_select_ties_go_to_the_lower_number(B, codes, span):  # noqa: F811
    import torch
    s = make(B, ([1, 20], [1600, 3000]), "bf16", 0, 2, 2, 64)
    g = torch.Generator("cuda").manual_seed(codes)
    k = random_bounds(s, g, span)
    k.codes.random_(-codes, codes + 1, generator=g)
    s.q.sign_()
    s.q[:, :, 3:] = 0
    check_select(s, k, 21, 1, 2)
    s.q.zero_()
    check_select(s, k, 21, 3, 1)


def test_select_strange_queries_and_bounds_that_were_never_written(B):  # noqa: F811
    import torch
    s = make(B, ([9], [2000]), "fp16", 0, 1, 2, 128)
    k = random_bounds(s, torch.Generator("cuda").manual_seed(5))
    s.q[0, 0, 5] = math.nan
    s.q[1, 1, 5] = math.inf
    s.q[2, 0] = -math.inf
    s.q[3] = 65504.0
    s.q[4] *= 2.0 ** -24
    s.q[5] = 255.0
    s.q[5, 0, 0] = 256.0
    k.codes[s.layer, s.host_table[0, 40:60].long()] = 0
    k.exps[s.layer, s.host_table[0, 40:60].long()] = 0
    check_select(s, k, 30, 1, 2)


@pytest.mark.parametrize("new,blocks,heads,n_blocks", [([1], 60000, 1, 100), ([1, 2], 20000, 2, 3000), ([1300], 6000, 2, 64), ([1], 700, 40, 7)])
def test_select_long(B, new, blocks, heads, n_blocks):  # noqa: F811
    """More scores than shared memory holds; long lists; more tokens than are in hand together; more heads than a warp."""
    import torch
    eng = B.Engine(n_layers=1, n_kv_heads=heads, head_dim=16, n_hbm_blocks=blocks, n_host_blocks=0, max_contexts=1, max_messages=16, max_tokens=64)
    g = torch.Generator("cuda").manual_seed(blocks)
    k = eng.key_bounds(torch.bfloat16)
    k.codes.random_(-127, 128, generator=g)
    k.exps.random_(120, 124, generator=g)
    n = len(new)
    table = torch.stack([torch.randperm(blocks, generator=g, device="cuda") for _ in new]).int()
    kv = [blocks * BT - 5 - 100 * i for i in range(n)]
    t = sum(new)
    q = torch.empty(t, heads * 2, 16, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    got = eng.select_blocks(0, q, k, table, ints([0, *np.cumsum(new)]), ints(kv), n_blocks).cpu().numpy()
    eng.kv_check()
    t0 = 0
    for i, m in enumerate(new):
        some = [0, m // 2, m - 1] if m > 3 else range(m)
        slots = table[i].long()
        want = lists_of(torch, q[[t0 + x for x in some]], k.codes[0, slots], k.exps[0, slots], [kv[i] - m + x for x in some], 2, n_blocks, 1, 2)
        assert np.array_equal(got[[t0 + x for x in some]], want)
        t0 += m


@pytest.mark.parametrize("codes,span", [(1, 1), (3, 2), (127, 1), (127, 4)])
@pytest.mark.parametrize("width,blocks", [(512, 500), (513, 513), (1024, 1000), (1025, 1025), (2048, 1500), (4096, 4000), (8192, 3000), (8192, 8192),
                                          (16384, 16000), (32768, 5000), (32768, 32768), (32769, 6000), (50000, 49999)])
def test_select_by_every_kernel(B, width, blocks, codes, span):  # noqa: F811
    """Scores that are the same many times over, and scores that hardly are, in rows of every length; short and long lists."""
    import torch
    eng = B.Engine(n_layers=1, n_kv_heads=2, head_dim=16, n_hbm_blocks=blocks, n_host_blocks=0, max_contexts=1, max_messages=16, max_tokens=64)
    g = torch.Generator("cuda").manual_seed(width + codes)
    k = eng.key_bounds(torch.bfloat16)
    k.codes.random_(-codes, codes + 1, generator=g)
    k.exps.random_(120, 120 + span, generator=g)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, :blocks] = torch.randperm(blocks, generator=g, device="cuda")
    q = torch.empty(3, 2, 16, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    if codes < 127:
        q.sign_()
        q[:, :, 4:] = 0
    q[2] = 0
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    for n_blocks, first, last in ((9, 1, 2), (64, 0, 1), (64, 5, 9), (300, 1, 2), (min(blocks - 1, 2000), 2, 2)):
        got = eng.select_blocks(0, q, k, table, ints(0, 3), ints(blocks * BT - 7), n_blocks, first=first, last=last).cpu().numpy()
        eng.kv_check()
        slots = table[0, :blocks].long()
        want = lists_of(torch, q, k.codes[0, slots], k.exps[0, slots], [blocks * BT - 10 + t for t in range(3)], 1, n_blocks, first, last)
        assert np.array_equal(got, want)


def test_selection_does_not_depend_on_the_batch(B):  # noqa: F811
    import torch
    s = make(B, ([30, 1, 17], [5000, 9000, 2000]), "bf16", 0, 2, 4, 128)
    k = random_bounds(s, torch.Generator("cuda").manual_seed(2), 2)
    whole = s.eng.select_blocks(1, s.q, k, s.table, s.q_start, s.kv_len, 33)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    t0 = 0
    for i, n in enumerate(s.new):
        for t in range(n):
            one = s.eng.select_blocks(1, s.q[t0 + t:t0 + t + 1], k, s.table[i:i + 1], ints(0, 1), ints(s.kv[i] - n + t + 1), 33)
            assert torch.equal(one[0], whole[t0 + t])
        t0 += n


# ---- attention over listed blocks ---------------------------------------------------------------
def random_lists(s, n, seed=0, holes=True, shuffle=True):
    """Up to n distinct blocks up to one behind each token's own, in any order, with entries that name nothing."""
    rng = np.random.default_rng(seed)
    out = np.full((s.rows, s.heads, n), -1, np.int32)
    t0 = 0
    for i, m in enumerate(s.new):
        for t in range(m):
            own = (s.kv[i] - m + t) // BT
            for h in range(s.heads):
                have = rng.permutation(own + 2)[:rng.integers(0, n + 1)]
                have = have if shuffle else np.sort(have)
                at = np.sort(rng.permutation(n)[:len(have)]) if holes else np.arange(len(have))
                out[t0 + t, h, at] = have
        t0 += m
    out[s.t:] = 0
    return s.torch.from_numpy(out).cuda()


def check_sparse(s, blocks, scale=None, want_lse=True, table=None):
    torch = s.torch
    hq, guard = s.heads * s.group, 7.25
    out = torch.full((s.rows, hq * 2, s.dim + 3), guard, dtype=s.dt, device="cuda")
    view = out[:, ::2, 1:1 + s.dim] if s.rows % 2 else out[:, :hq, :s.dim]
    lse = torch.full((s.rows, hq), guard, device="cuda") if want_lse else None
    before = s.bits()
    s.eng.attend_blocks(s.layer, s.q, blocks, s.table if table is None else table, s.q_start, s.kv_len, scale=scale, out=view, lse=lse)
    s.eng.kv_check()
    want, wl, tol, tl = sparse_reference(s, blocks, scale)
    got = view[:s.t].double()
    assert bool(torch.isfinite(got).all())
    assert not bool(((got - want).abs() > tol).any()), float(((got - want).abs() - tol).max())
    assert bool((view[s.t:] == guard).all())
    if want_lse:
        none = torch.isinf(wl)
        assert torch.equal(torch.isinf(lse[:s.t]), none) and bool((got[none] == 0).all())
        assert not bool(((lse[:s.t].double() - wl).abs() > tl)[~none].any())
        assert bool((lse[s.t:] == guard).all())
    assert all(torch.equal(a, b) for a, b in zip(before, s.bits()))


@pytest.mark.parametrize("n", [1, 6, 33])
@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("dtype,layout,heads,group,dim", HEADS)
def test_attend_blocks(B, batch, dtype, layout, heads, group, dim, n):  # noqa: F811
    s = make(B, batch, dtype, layout, heads, group, dim, tail=n == 6, pad=n % 3, strided=n == 33)
    check_sparse(s, random_lists(s, n, seed=n), want_lse=n != 6, scale=0.3 if n == 1 else None)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [1, 4, 5, 8, 9, 16, 20])
@pytest.mark.parametrize("dim", [64, 128, 40, 96, 200])
@pytest.mark.parametrize("n,new", [(200, [1]), (64, [1, 1, 2]), (17, [40, 7]), (130, [3, 60])])
def test_attend_blocks_groups(B, dtype, group, dim, n, new):  # noqa: F811
    """Clusters of every size, CTAs and warps per unit."""
    s = make(B, (new, [4000, 1000, 70][:len(new)]), dtype, 0, 2, group, dim, layers=1, layer=0)
    check_sparse(s, random_lists(s, n, seed=group, holes=False, shuffle=False))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [1, 4, 7, 8, 12, 18])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_blocks_of_many_tokens(B, dtype, group, dim):  # noqa: F811
    """More units than warps run at once, empty lists among them, a sequence behind whose tokens there are rows of nobody."""
    s = make(B, ([600, 33], [300, 20]), dtype, 0, 2, group, dim, layers=1, layer=0, pad=3, tail=group == 4, strided=group == 7, q_gain=2.0)
    check_sparse(s, random_lists(s, 7, seed=group))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [2, 8])
def test_attend_blocks_scores_that_climb_and_fall(B, dtype, group):  # noqa: F811
    import torch
    s = make(B, ([1, 30], [3000, 2000]), dtype, 0, 1, group, 128, layers=1, layer=0)
    for i in range(2):
        for b in range(s.kv[i] // BT):
            x = s._chunk(int(s.host_table[i, b]), 0)
            x.mul_(0.1 + 6 * abs(math.sin(b / 9)))
    check_sparse(s, random_lists(s, 90, seed=3, holes=False))


def test_attend_blocks_listed_blocks_alone_count(B):  # noqa: F811
    """NaN and Inf in blocks that are not listed, behind the token, and in rows of other tokens."""
    import torch
    s = make(B, ([20, 1], [400, 333]), "bf16", 0, 2, 4, 64)
    lists = random_lists(s, 9, seed=4)
    lists[lists == 3] = 4
    lists[0, 0] = torch.tensor([5, 3, -1, -5, 7, 2 ** 31 - 1, -2 ** 31, 1, 0], device="cuda")
    bad = int(s.host_table[0, 3])
    for c in (0, 1):
        s._chunk(bad, c).fill_(math.nan)
    want = s.eng.attend_blocks(s.layer, s.q, torch.where(lists == 3, -1, lists).int(), s.table, s.q_start, s.kv_len)
    got = s.eng.attend_blocks(s.layer, s.q, lists, s.table, s.q_start, s.kv_len)
    s.eng.kv_check()
    assert torch.equal(want[1:], got[1:]) and torch.equal(want[0, 4:], got[0, 4:])
    assert bool(torch.isfinite(want).all()) and bool(torch.isnan(got[0, :4]).all())


def test_attend_blocks_over_all_blocks_is_attend(B):  # noqa: F811
    import torch
    s = make(B, ([1, 37, 64], [700, 300, 0]), "bf16", 1, 2, 4, 128, tail=True)
    n = s.table.shape[1]
    every = torch.arange(n, dtype=torch.int32, device="cuda").expand(s.t, 2, n).contiguous()
    a = s.eng.attend_blocks(s.layer, s.q, every, s.table, s.q_start, s.kv_len)
    want, _, tol, _ = s.reference()
    assert not bool(((a.double() - want).abs() > tol).any())


# ---- weights ------------------------------------------------------------------------------------
def check_weigh(s, window=0, causal=True, scale=None, keep=None, hint=True, in_place=False):
    torch = s.torch
    lse = torch.empty(s.rows, s.heads * s.group, device="cuda")
    s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len, window=window, causal=causal, scale=scale, lse=lse)
    g = torch.Generator("cuda").manual_seed(9)
    wide = torch.rand(len(s.new), s.table.shape[1] + 3, generator=g, device="cuda").mul_(3)[:, 1:-2]
    old = wide.clone() if keep is not None else None
    for hint in (max(s.new + [1]), None, 1):
        out = old.clone() if in_place else None
        given = out if in_place else old
        got = s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len, max_q_len=hint, window=window, causal=causal, scale=scale,
                                 weights=given, keep=keep if keep is not None else 1.0, out=out)
        s.eng.kv_check()
        want, tol = weights_reference(s, lse, window, causal, scale)
        if keep is not None:
            held = torch.arange(s.table.shape[1], device="cuda") * BT < s.kv_len[:, None]
            want = torch.where(held, want + float(np.float32(keep)) * old.double(), 0.0)
        assert bool(torch.isfinite(got).all())
        assert not bool(((got.double() - want).abs() > tol + 4 * E32 * want.abs()).any()), float(((got.double() - want).abs() / (tol + 1e-30)).max())
    return got


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("dtype,layout,heads,group,dim", HEADS)
def test_weigh(B, batch, dtype, layout, heads, group, dim):  # noqa: F811
    s = make(B, batch, dtype, layout, heads, group, dim, tail=True, pad=2, strided=heads == 2, q_gain=3.0)
    check_weigh(s, keep=0.75)


@pytest.mark.parametrize("dim", [64, 128, 24])
@pytest.mark.parametrize("batch", ["step", "ragged", "fills", ([300], [500]), ([130, 1, 5], [0, 40, 4000])])
@pytest.mark.parametrize("window", [1, 16, 100, 5000])
def test_weigh_window(B, batch, window, dim):  # noqa: F811
    check_weigh(make(B, batch, "bf16", 0, 2, 2, dim), window=window, scale=0.2)


@pytest.mark.parametrize("new", [[1, 1], [90, 3]])
def test_weigh_blocks_in_front_of_the_window_need_no_slot(B, new):  # noqa: F811
    import torch
    s = make(B, (new, [1000, 5000]), "bf16", 0, 2, 4, 64)
    want = check_weigh(s, window=200)
    for i, n in enumerate(new):
        s.table[i, :(s.kv[i] - n + 1 - 200) // BT] = -1
    lse = torch.empty(s.rows, 8, device="cuda")
    s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len, window=200, lse=lse)
    got = s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len, max_q_len=1, window=200)
    s.eng.kv_check()
    assert torch.equal(got, want)
    got = s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len, window=200)
    s.eng.kv_check()
    assert torch.allclose(got, want, rtol=1e-5, atol=0)


@pytest.mark.parametrize("dim", [64, 128, 40])
@pytest.mark.parametrize("batch", [*BATCHES, ([200, 3], [100, 900])])
def test_weigh_full(B, batch, dim):  # noqa: F811
    check_weigh(make(B, batch, "fp16", 0, 1, 3, dim), causal=False, keep=1.0, in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,heads,group", [(128, 2, 4), (64, 4, 3), (128, 1, 12), (64, 3, 1), (128, 1, 40), (64, 1, 130)])
@pytest.mark.parametrize("new,past", [([600], [0]), ([257, 1, 40], [1000, 3000, 17]), ([64], [5000]), ([1000, 129], [77, 2000])])
def test_weigh_prompts_and_chunks(B, dtype, dim, heads, group, new, past):  # noqa: F811
    s = make(B, (new, past), dtype, 0, heads, group, dim, layers=1, layer=0, q_gain=2.0, tail=group == 3, strided=group == 12)
    check_weigh(s)


@pytest.mark.parametrize("dim,group", [(128, 4), (64, 7), (40, 2)])
def test_many_sequences(B, dim, group):  # noqa: F811
    """More of them than a warp has lanes, some without new tokens, some without any."""
    import torch
    n = 75
    new, past = [(i * 7) % 45 if i % 6 else 0 for i in range(n)], [(i * 131) % 900 if i % 5 else 0 for i in range(n)]
    s = make(B, (new, past), "bf16", 0, 2, group, dim, layers=1, layer=0, tail=True, pad=5)
    check_bounds(s)
    k = random_bounds(s, torch.Generator("cuda").manual_seed(3))
    check_select(s, k, 9, 1, 2)
    check_sparse(s, random_lists(s, 4, seed=5))
    check_weigh(s, keep=0.5)
    check_weigh(s, window=70)


@pytest.mark.parametrize("new,past,window", [([40, 1], [30000, 9000], 0), ([64, 3], [20000, 100], 9000), ([9], [66000], 0)])
def test_weigh_long(B, new, past, window):  # noqa: F811
    check_weigh(make(B, (new, past), "bf16", 0, 1, 4, 64, layers=1, layer=0), window=window)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("scale,gain", [(1e-3, 4.0), (4.0, 1.0), (0.125, 30.0), (5e-5, 1.0), (3e4, 1e-3), (0.0, 1.0), (1.0, 8.0)])
def test_weigh_scales_near_and_far(B, dtype, scale, gain):  # noqa: F811
    """lse of some thousands and of nearly nothing."""
    for new in ([200], [2]):
        s = make(B, (new, [300]), dtype, 0, 2, 4, 128, layers=1, layer=0, q_gain=gain)
        check_weigh(s, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lse", [5.0, 3e8, 6e9, 2e11, 1e28, 3e38, -3e8, -6e9, -2e11, -1e28, -3e38, math.inf, math.nan])
def test_weigh_lse_of_any_size(B, dtype, dim, lse):  # noqa: F811
    """Scores of 0 and of +- 2^29 dim / sqrt(dim), the same by every kernel: far from lse, so that every weight is 0 or Inf, or at 0."""
    import torch
    s = make(B, ([60], [500]), dtype, 0, 1, 2, dim, layers=1, layer=0)
    s.q.fill_(2.0 ** 15)
    for b in range(s.host_table.shape[1] - 2):
        s._chunk(int(s.host_table[0, b]), 0).fill_((0.0, 2.0 ** 14, -2.0 ** 14)[b % 3])
    rows = torch.full((s.t, 2), lse, device="cuda")
    rows[::2] = -math.inf                   # half of the rows count for nothing
    n = s.table.shape[1]
    want = torch.zeros(n, dtype=torch.float64)
    for b in range(n - 2):
        score = (0.0, 1.0, -1.0)[b % 3] * 2.0 ** 29 * dim ** 0.5
        for i in range(b * BT, min(b * BT + BT, s.kv[0])):
            seen = sum(1 for t in range(1, s.t, 2) if 500 + t >= i)
            if seen:
                x = score - float(np.float32(lse))
                want[b] += 2 * seen * (math.nan if math.isnan(x) else math.inf if x > 700 else math.exp(x))
    want = want.float().double()
    for hint in (None, 1):
        got = s.eng.weigh_blocks(0, s.q, rows, s.table, s.q_start, s.kv_len, max_q_len=hint)[0].double().cpu()
        s.eng.kv_check()
        fine = torch.isfinite(want)
        assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]) and torch.equal(torch.isnan(got), torch.isnan(want))
        # at a score of 0 and lse of 5: powers to 2^-22 and 5 * 2^-22, and 32-bit sums
        assert bool(((got - want).abs()[fine] <= want[fine] * (6 * 2.0 ** -22 + (n * 40) * E32)).all())


def test_weights_sum_to_the_number_of_rows(B):  # noqa: F811
    s = make(B, ([50, 1, 700], [10, 5000, 0]), "bf16", 0, 2, 4, 128)
    got = check_weigh(s).double().sum(1).cpu()
    for i, n in enumerate(s.new):
        assert abs(float(got[i]) / (n * 8) - 1) < 2e-5


def test_weigh_rows_without_keys_and_masked_nan(B):  # noqa: F811
    """lse of -inf adds nothing, whatever the keys; keys behind a token have no effect."""
    import torch
    for new in ([40], [1], [300]):
        s = make(B, (new, [100]), "bf16", 0, 2, 2, 64)
        lse = torch.full((s.t, 4), -math.inf, device="cuda")
        got = s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len)
        assert bool((got == 0).all())
        check_weigh(s)
        last = s.kv[0] - 1                 # a NaN key that the last token alone sees
        s._chunk(int(s.host_table[0, last // BT]), 0)[last % BT].fill_(math.nan)
        lse = torch.full((s.t, 4), 3.0, device="cuda")
        lse[-1] = -math.inf
        got = s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len)
        assert not bool(torch.isnan(got[:, :last // BT]).any())


@pytest.mark.parametrize("new,dim,hint", [(65536, 64, None), (65536, 128, None), (65536, 64, 1), (40000, 40, None)])
def test_weigh_long_prompts_lose_nothing(B, new, dim, hint):  # noqa: F811
    """All scores 0 and lse the same, so that every key gets exp(-lse) from every row that sees it. However many rows there are, the result is off
    by the power (2^-22, and the exponent by 4 * 3.7 * 2^-24) and by what sums of up to 80 powers lose in 32 bits (80 * 2^-24)."""
    import torch
    s = make(B, ([new], [0]), "bf16", 0, 2, 4, dim, layers=1, layer=0)
    s.q.zero_()
    lse = torch.full((new, 8), 3.7, device="cuda")
    got = s.eng.weigh_blocks(0, s.q, lse, s.table, s.q_start, s.kv_len, max_q_len=hint)[0, :new // BT].double().cpu().numpy()
    s.eng.kv_check()
    rows = (new - np.arange(new)).reshape(-1, BT).sum(1) * 8.0
    want = rows * math.exp(-float(np.float32(3.7)))
    assert float(np.abs(got / want - 1).max()) <= 2.0 ** -22 + 4 * 3.7 * E32 + 80 * E32


def test_weigh_adds_the_layers_up(B):  # noqa: F811
    import torch
    s = make(B, ([3, 1], [200, 90]), "bf16", 0, 2, 4, 64, layers=2, layer=0)
    lse = torch.full((s.t, 8), 4.0, device="cuda")
    first = s.eng.weigh_blocks(0, s.q, lse, s.table, s.q_start, s.kv_len)
    both = s.eng.weigh_blocks(0, s.q, lse, s.table, s.q_start, s.kv_len, weights=first)
    assert torch.allclose(both, 2 * first, rtol=1e-6, atol=0)


def test_weigh_is_the_same_every_time(B):  # noqa: F811
    import torch
    for new, past in (([1, 1], [4000, 900]), ([700], [300]), ([40, 3], [2000, 10])):
        s = make(B, (new, past), "bf16", 0, 2, 4, 128)
        lse = torch.full((s.t, 8), 5.0, device="cuda")
        runs = [s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len) for _ in range(4)]
        assert all(torch.equal(runs[0], r) for r in runs[1:])


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("strided", [False, True])
def test_weigh_that_gives_up_a_wait_writes_nothing(B, dtype, dim, strided):  # noqa: F811
    """40 and 33 tokens on long contexts: a CTA has more jobs than it holds at once, so its planning warp has to wait. Where that wait runs
    out the call ends, says so, and leaves the weights that it was given as they were, whatever was in its scratch before."""
    import torch
    s = make(B, ([40, 33], [100000, 60000]), dtype, 0, 2, 2, dim, layers=1, layer=0, strided=strided)
    lse = torch.full((s.rows, 4), 6.0, device="cuda")
    old = torch.rand(s.table.shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    call = lambda w: s.eng.weigh_blocks(s.layer, s.q, lse, s.table, s.q_start, s.kv_len, weights=w, out=w)      # noqa: E731
    want = call(old.clone())
    s.eng.kv_check()
    weights = old.clone()
    s.eng.set_wait_limit(0)
    b = B.Batch(*s.eng._kv_batch("", s.t, s.table, s.q_start, s.kv_len, 0))
    a = B.WeighArgs(b, 0, 0 if dtype == "bf16" else 1, 4, 0, 0, 0.0, 1.0, 0, s.q.data_ptr(), lse.data_ptr(), *s.q.stride()[:2], weights.data_ptr(),
                    weights.data_ptr(), weights.stride(0), weights.stride(0), 0, 0)
    n = s.eng.L.kvt_weigh_scratch_bytes(s.eng.h, C.byref(a))
    assert n
    scratch = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    a.scratch, a.scratch_bytes = scratch.data_ptr(), n
    assert s.eng.L.kvt_weigh_blocks(s.eng.h, C.byref(a), s.eng._kv_stream()) == 0
    with pytest.raises(B.KvtError, match="wait"):
        s.eng.kv_check()
    assert torch.equal(weights, old)
    s.eng.set_wait_limit(1 << 18)
    scratch.fill_(255)
    assert s.eng.L.kvt_weigh_blocks(s.eng.h, C.byref(a), s.eng._kv_stream()) == 0
    s.eng.kv_check()
    assert torch.equal(weights, want)


# ---- eviction -----------------------------------------------------------------------------------
def evict_reference(table, weights, kv_len, n_blocks, first, last):
    t, w, e, n = np.full_like(table, -1), np.zeros_like(weights), np.full_like(table, -1), kv_len.copy()
    for i, kv in enumerate(kv_len):
        had = -(-int(kv) // BT)
        free = list(range(first, max(first, had - last))) if had > n_blocks else []
        free.sort(key=lambda b: (np.inf if np.isnan(weights[i, b]) else weights[i, b], -b))
        gone = sorted(free[:max(0, had - n_blocks)])
        kept = np.setdiff1d(np.arange(had), gone).astype(int)
        t[i, :len(kept)], w[i, :len(kept)], e[i, :len(gone)] = table[i, kept], weights[i, kept], table[i, gone]
        n[i] = kv - BT * len(gone)
    return t, n, w, e


@pytest.mark.parametrize("n_blocks,first,last", [(40, 1, 2), (3, 0, 1), (7, 3, 4), (5000, 4, 32), (100000, 1, 2)])
@pytest.mark.parametrize("kv,width", [([0, 1, 16, 700, 9999], 700), ([100000], 6250), ([1000003, 640, 5], 62501), ([639, 640, 641, 656, 657], 45), ([65540, 70000, 100], 4376),
                                      ([400000, 524288], 32768), ([2200001], 137501)])
@pytest.mark.parametrize("values", ["random", "few", "strange", "near"])
def test_evict(B, kv, width, n_blocks, first, last, values):  # noqa: F811
    import torch
    eng = B.Engine(n_layers=1, n_kv_heads=1, head_dim=64, n_hbm_blocks=4, n_host_blocks=0, max_contexts=1, max_messages=16, max_tokens=64)
    g = torch.Generator("cuda").manual_seed(width + n_blocks)
    n = len(kv)
    table = torch.randint(0, 2 ** 31 - 1, (n, width + 3), generator=g, device="cuda", dtype=torch.int32)[:, 2:-1]
    weights = torch.randn(n, width + 1, generator=g, device="cuda")[:, 1:]
    if values == "few":
        weights = weights.mul_(1.5).round_()
    if values == "near":                     # apart in the last of the 32 bits alone: most of them, and of the rest, three by three, two alike and one next to them
        weights = weights.mul_(20).round_() * 2.0 ** -23 + 1
        rest = torch.randn(n, -(-width // 9), generator=g, device="cuda") * 2
        for i, x in ((0, rest), (3, rest), (6, torch.nextafter(rest, torch.full_like(rest, math.inf)))):
            weights[:, i::9] = x[:, :weights[:, i::9].shape[1]]
    if values == "strange":
        weights[:, ::7] = math.nan
        weights[:, ::5] = -math.inf
        weights[:, 2::11] = math.inf
        weights[:, 3::13] = -0.0
        weights[:, 4::13] = 0.0
    kv_len = torch.tensor(kv, dtype=torch.int32, device="cuda")
    want = evict_reference(table.cpu().numpy(), weights.cpu().numpy(), kv_len.cpu().numpy(), n_blocks, first, last)

    def check(got):
        for x, y in zip(got, want):
            assert np.array_equal(x.cpu().numpy(), y, equal_nan=x.is_floating_point())

    check(eng.evict_blocks(weights, table, kv_len, n_blocks, first=first, last=last))
    eng.kv_check()
    evicted = torch.empty(n, width, dtype=torch.int32, device="cuda")
    check(eng.evict_blocks(weights, table, kv_len, n_blocks, first=first, last=last, out=(table, kv_len, weights, evicted)))


# ---- errors, streams, graphs --------------------------------------------------------------------
def test_bad_slots_and_lengths_are_reported_and_harmless(B):  # noqa: F811
    import torch
    for new in ([1, 20], [30, 300]):
        s = make(B, (new, [400, 300]), "bf16", 0, 2, 2, 64, tail=True)
        k = random_bounds(s, torch.Generator("cuda").manual_seed(1))
        lists = torch.arange(26, dtype=torch.int32, device="cuda").expand(s.t, 2, 26).contiguous()
        lse = torch.full((s.t, 4), 5.0, device="cuda")
        ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
        t = s.t
        far = s.table.clone()
        far[1, 5], far[1, 9], far[0, 24] = -1, 0x7FFFFFF0, 1 << 20
        calls = {"slot": (far, s.q_start, s.kv_len), "length": (s.table, s.q_start, ints(s.kv[0], 1 << 30)), "negative": (s.table, s.q_start, ints(-5, 300)),
                 "short": (s.table, s.q_start, ints(0, 10)), "starts": (s.table, ints(0, t, 5), s.kv_len), "behind": (s.table, ints(0, 5, t + 100), s.kv_len),
                 "both ways": (s.table, ints(t, 3, t), s.kv_len)}
        for name, batch in calls.items():
            before = s.bits()
            ops = {"bound": lambda: s.eng.bound_keys(1, k, *batch, n_tokens=t), "select": lambda: s.eng.select_blocks(1, s.q, k, *batch, 9),
                   "attend": lambda: s.eng.attend_blocks(1, s.q, lists, *batch), "weigh": lambda: s.eng.weigh_blocks(1, s.q, lse, *batch)}
            for op, call in ops.items():
                call()
                if name == "slot" and op == "bound":      # the slots in question are not those of a block that is filled
                    s.eng.kv_check()
                elif name == "short" and op == "weigh":   # a length that holds less than its new tokens: those without a place see nothing
                    s.eng.kv_check()
                else:
                    with pytest.raises(B.KvtError):
                        s.eng.kv_check()
                s.eng.kv_check()
            assert all(torch.equal(a, b) for a, b in zip(before, s.bits()))
        with pytest.raises(B.KvtError):
            s.eng.evict_blocks(torch.zeros(2, 5, device="cuda"), s.table[:, :5].contiguous(), ints(81, 80), 3)
            s.eng.kv_check()


def test_refusals(B):  # noqa: F811
    import torch
    s = make(B, ([3, 1], [200, 90]), "bf16", 0, 2, 4, 64)
    k = s.eng.key_bounds(torch.bfloat16)
    batch = (s.table, s.q_start, s.kv_len)
    lse = torch.zeros(s.t, 8, device="cuda")
    lists = torch.zeros(s.t, 2, 5, dtype=torch.int32, device="cuda")
    w = torch.zeros(s.table.shape, device="cuda")
    eng, q, layer = s.eng, s.q, s.layer
    bad = (ValueError, B.KvtError)

    def no(call):
        with pytest.raises(bad):
            call()

    for lay in (-1, 2):
        no(lambda: eng.bound_keys(lay, k, *batch, n_tokens=4))
        no(lambda: eng.select_blocks(lay, q, k, *batch, 5))
        no(lambda: eng.attend_blocks(lay, q, lists, *batch))
        no(lambda: eng.weigh_blocks(lay, q, lse, *batch))
    for wrong in (q.half(), q.float(), q[:, :7], q[:, :, :32], q[:3], q.cpu(), q.transpose(1, 2), q[:, :0]):
        no(lambda: eng.attend_blocks(layer, wrong, lists, *batch) if wrong.dtype != torch.float16 else eng.select_blocks(layer, wrong, k, *batch, 5))
        no(lambda: eng.weigh_blocks(layer, wrong if wrong.dtype != torch.float16 else q[:, :7], lse, *batch))
    for n, first, last in ((0, 0, 0), (5, 0, 0), (5, 4, 2), (5, -1, 2), (-3, 1, 2)):
        no(lambda: eng.select_blocks(layer, q, k, *batch, n, first=first, last=last))
        no(lambda: eng.evict_blocks(w, s.table, s.kv_len, n, first=first, last=last))
    other = B.KeyBounds(torch.bfloat16, k.codes[:, :, :1].contiguous(), k.exps[:, :, :1].contiguous())
    for x in (other, B.KeyBounds(torch.float16, k.codes, k.exps), B.KeyBounds(torch.bfloat16, k.codes.cpu(), k.exps), B.KeyBounds(torch.bfloat16, k.codes, k.exps.int())):
        no(lambda: eng.select_blocks(layer, q, x, *batch, 5))
    no(lambda: eng.bound_keys(layer, other, *batch, n_tokens=4))
    no(lambda: eng.bound_keys(layer, k, *batch, n_tokens=-1))
    no(lambda: eng.key_bounds(torch.float32))
    for x in (lists.long(), lists[:3], lists[:, :1], lists.cpu(), lists[:, :, ::2], lists[0], lists[:, :, :0]):
        no(lambda: eng.attend_blocks(layer, q, x, *batch))
    for x in (lse.double(), lse[:3], lse[:, :7], lse.cpu(), lse.T.contiguous().T):
        no(lambda: eng.weigh_blocks(layer, q, x, *batch))
        no(lambda: eng.attend_blocks(layer, q, lists, *batch, lse=x))
    for x in (w[:, :3], w.double(), w.cpu(), w.T.contiguous().T):
        no(lambda: eng.weigh_blocks(layer, q, lse, *batch, weights=x))
        no(lambda: eng.weigh_blocks(layer, q, lse, *batch, out=x))
        no(lambda: eng.evict_blocks(x, s.table, s.kv_len, 5))
    no(lambda: eng.weigh_blocks(layer, q, lse, *batch, out=w[:1].expand(2, -1)))
    no(lambda: eng.weigh_blocks(layer, q, lse, *batch, weights=w[:1].expand(2, -1), out=w))
    for kw in (dict(keep=-1.0), dict(keep=math.nan), dict(keep=math.inf), dict(scale=-1.0), dict(scale=math.nan), dict(window=-1),
               dict(window=5, causal=False), dict(max_q_len=-1)):
        no(lambda: eng.weigh_blocks(layer, q, lse, *batch, weights=w, **kw))
    for scale in (-1.0, math.nan, math.inf):
        no(lambda: eng.attend_blocks(layer, q, lists, *batch, scale=scale))
    no(lambda: eng.attend_blocks(layer, q, lists, *batch, out=q[:1].expand(4, 8, 64)))
    for i in range(3):
        wrong = list(batch)
        for x in (wrong[i].long(), wrong[i].cpu(), wrong[i][:1]):
            wrong[i] = x
            no(lambda: eng.bound_keys(layer, k, *wrong, n_tokens=4))
            no(lambda: eng.select_blocks(layer, q, k, *wrong, 5))
            no(lambda: eng.attend_blocks(layer, q, lists, *wrong))
            no(lambda: eng.weigh_blocks(layer, q, lse, *wrong))
    e = torch.empty_like(s.table)
    no(lambda: eng.evict_blocks(w, s.table, s.kv_len, 5, out=(s.table, s.kv_len, w, s.table)))
    no(lambda: eng.evict_blocks(w, s.table, s.kv_len, 5, out=(s.table, s.kv_len.long(), w, e)))
    no(lambda: eng.evict_blocks(w, s.table, s.kv_len[:1], 5))
    no(lambda: eng.evict_blocks(w, s.table.long(), s.kv_len, 5))
    no(lambda: eng.evict_blocks(w, s.table, s.kv_len, 5, out=(e[:1].expand(2, -1), s.kv_len, w, s.table)))
    grad = q.float().requires_grad_().bfloat16()
    for call in (lambda: eng.select_blocks(layer, grad, k, *batch, 5), lambda: eng.attend_blocks(layer, grad, lists, *batch),
                 lambda: eng.weigh_blocks(layer, grad, lse, *batch), lambda: eng.weigh_blocks(layer, q, lse.clone().requires_grad_(), *batch),
                 lambda: eng.weigh_blocks(layer, q, lse, *batch, weights=w.clone().requires_grad_())):
        no(call)
        with torch.no_grad():
            call()
    s.eng.kv_check()
    meta = B.Engine(n_layers=1, n_kv_heads=2, head_dim=64, n_hbm_blocks=4, n_host_blocks=0, max_contexts=1, metadata_only=True)
    no(lambda: meta.attend_blocks(0, q, lists, *batch))
    no(lambda: meta.key_bounds(torch.bfloat16))


def test_scratch_that_is_too_small_or_misaligned(B):  # noqa: F811
    import torch
    s = make(B, ([40], [3000]), "bf16", 0, 2, 4, 64)
    k = s.eng.key_bounds(torch.bfloat16)
    kb = s.eng._bounds("", k)
    out = torch.empty(s.t, 2, 9, dtype=torch.int32, device="cuda")
    b = B.Batch(*s.eng._kv_batch("", s.t, s.table, s.q_start, s.kv_len, 40))
    a = B.SelectArgs(b, 1, 0, 8, 9, 1, 2, s.q.data_ptr(), *s.q.stride()[:2], kb, out.data_ptr(), 0, 0)
    n = s.eng.L.kvt_select_scratch_bytes(s.eng.h, C.byref(a))
    room = torch.empty(n + 16, dtype=torch.uint8, device="cuda")
    call = lambda: s.eng.L.kvt_select_blocks(s.eng.h, C.byref(a), s.eng._kv_stream())      # noqa: E731
    assert call() == B.E_BUFSZ
    a.scratch, a.scratch_bytes = room.data_ptr(), n - 1
    assert call() == B.E_BUFSZ
    a.scratch, a.scratch_bytes = room.data_ptr() + 4, n
    assert call() == B.E_INVAL
    a.scratch = room.data_ptr() + 16
    assert call() == 0
    want = s.eng.select_blocks(1, s.q, k, s.table, s.q_start, s.kv_len, 9)
    s.eng.kv_check()
    assert torch.equal(out, want)


def test_nothing_to_do(B):  # noqa: F811
    import torch
    s = make(B, ([3, 1], [200, 90]), "bf16", 0, 2, 4, 64)
    k = s.eng.key_bounds(torch.bfloat16)
    none = (s.table[:0], s.q_start[:1], s.kv_len[:0])
    q, lse = s.q[:0], torch.zeros(0, 8, device="cuda")
    lists = torch.zeros(0, 2, 5, dtype=torch.int32, device="cuda")
    for batch in (none, (s.table, torch.zeros_like(s.q_start), s.kv_len)):
        s.eng.bound_keys(0, k, *batch, n_tokens=0)
        assert s.eng.select_blocks(0, q, k, *batch, 5).shape == (0, 2, 5)
        assert s.eng.attend_blocks(0, q, lists, *batch).shape == (0, 8, 64)
    assert s.eng.weigh_blocks(0, q, lse, *none).shape == (0, s.table.shape[1])
    w = torch.rand(s.table.shape, device="cuda")
    got = s.eng.weigh_blocks(0, q, lse, s.table, torch.zeros_like(s.q_start), s.kv_len, weights=w, keep=0.5)
    held = torch.arange(s.table.shape[1], device="cuda") * BT < s.kv_len[:, None]
    assert torch.equal(got, torch.where(held, w * 0.5, 0.0))
    assert s.eng.evict_blocks(w[:0], *none[::2], 5)[0].shape == none[0].shape
    s.eng.kv_check()


def test_native_and_python_marshalling_make_the_same_call(B, monkeypatch):  # noqa: F811
    import torch
    s = make(B, ([40, 1], [900, 2000]), "bf16", 0, 2, 4, 64, tail=True, strided=True)
    batch = (s.table, s.q_start, s.kv_len)
    lse = torch.full((s.t, 8), 6.0, device="cuda")
    old = torch.rand(s.table.shape, device="cuda")

    def run():
        k = s.eng.key_bounds(s.dt)
        s.eng.bound_keys(s.layer, k, *batch, n_tokens=s.t)
        k.codes.random_(-127, 128, generator=torch.Generator("cuda").manual_seed(1))
        k.exps.fill_(120)
        blocks = s.eng.select_blocks(s.layer, s.q, k, *batch, 12, first=2, last=3, max_q_len=40)
        return (k.codes, blocks, s.eng.attend_blocks(s.layer, s.q, blocks, *batch, scale=0.25, lse=torch.empty_like(lse)),
                s.eng.weigh_blocks(s.layer, s.q, lse, *batch, max_q_len=40, window=500, scale=0.25, weights=old, keep=0.5),
                *s.eng.evict_blocks(old, s.table, s.kv_len, 20, first=3, last=4))

    want = run()
    for name in ("bound", "select", "attend_blocks", "weigh", "evict"):
        assert s.eng.__dict__[f"_{name}_native"] is not None
        monkeypatch.setattr(s.eng, f"_{name}_native", lambda *args: NotImplemented)
    for x, y in zip(want, run()):
        assert torch.equal(x, y)
    s.eng.kv_check()


def whole_step(s, k, weights, budget=9):
    """The set as a step of a serving loop runs it."""
    eng, batch = s.eng, (s.table, s.q_start, s.kv_len)
    eng.bound_keys(s.layer, k, *batch, n_tokens=s.t)
    blocks = eng.select_blocks(s.layer, s.q, k, *batch, budget)
    out = eng.attend_blocks(s.layer, s.q, blocks, *batch)
    lse = s.torch.empty(s.t, s.heads * s.group, device="cuda")
    eng.attend(s.layer, s.q, *batch, lse=lse)
    eng.weigh_blocks(s.layer, s.q, lse, *batch, weights=weights, out=weights)
    return (blocks, out, weights, *eng.evict_blocks(weights, s.table, s.kv_len, budget))


@pytest.mark.parametrize("new,past", [([1, 1, 1], [900, 300, 15]), ([200, 3], [700, 2000])])
def test_captured_and_replayed_with_other_lengths(B, new, past):  # noqa: F811
    import torch
    s = make(B, (new, past), "bf16", 0, 2, 4, 64)
    k = random_bounds(s, torch.Generator("cuda").manual_seed(3))
    w = torch.zeros(s.table.shape, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        whole_step(s, k, w)
    torch.cuda.current_stream().wait_stream(side)
    graphs, results = [], []
    for _ in range(2):                       # two graphs of the same calls, one of which runs while the other's results are in use
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(whole_step(s, k, w))
        graphs.append(graph)
    for lengths in (s.kv, [n - 17 for n in s.kv], [s.kv[0], *[n - 40 for n in s.kv[1:]]]):
        if min(n - m for n, m in zip(lengths, s.new)) < 0:
            continue
        s.kv_len.copy_(torch.tensor(lengths, dtype=torch.int32))
        w.zero_()
        want = [x.clone() for x in whole_step(s, k, w)]
        for graph, got in zip(graphs, results):
            w.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(want, got))
    s.eng.kv_check()


def test_two_streams_at_once(B):  # noqa: F811
    import torch
    s = [make(B, (n, p), "bf16", 0, 2, 4, 128, seed=i) for i, (n, p) in enumerate([([1, 1], [5000, 300]), ([60], [4000])])]
    k = [random_bounds(x, torch.Generator("cuda").manual_seed(3)) for x in s]
    zeros = lambda x: torch.zeros(x.table.shape, device="cuda")      # noqa: E731
    want = [whole_step(x, y, zeros(x)) for x, y in zip(s, k)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = whole_step(s[i], k[i], zeros(s[i]))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


# ---- the set as it is used ----------------------------------------------------------------------
@pytest.mark.parametrize("layout", [0, 1])
def test_long_session_with_sparse_steps_and_eviction(B, layout):  # noqa: F811
    """A context's prompt is appended, bounded, attended to and weighed; steps attend to some of its blocks; the lightest blocks leave
    its table and go back to the engine; its next steps go on at their old positions over what stayed."""
    import torch
    dt, hq, dim = torch.bfloat16, 6, 64
    eng = B.Engine(n_layers=2, n_kv_heads=2, head_dim=dim, n_hbm_blocks=90, n_host_blocks=4, max_contexts=4, max_messages=64, max_tokens=4096,
                   pool_layout=layout, n_tail_blocks=3)
    g = torch.Generator("cuda").manual_seed(layout)
    rope = B.Rope(dim)
    bounds = eng.key_bounds(dt)
    eng.spawn(0)
    eng.append(0, np.arange(1000, dtype=np.uint32))
    eng.map_blocks([0], B.MAP_LOOKUP)
    eng.map_blocks([0], B.MAP_ADMIT)
    _, tier, slot = eng.get_block_map(0)
    assert len(slot) == 62 and bool((tier == B.TIER_HBM).all())
    table = torch.full((1, 70), -1, dtype=torch.int32, device="cuda")
    table[0, :62] = torch.from_numpy(slot.astype(np.int32))
    table[0, 62] = eng.n_hbm_blocks            # the partly filled block
    weights = torch.zeros(1, 70, device="cuda")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    freqs = [10000.0 ** (-2 * j / dim) for j in range(dim // 2)]
    caches = [eng.hbm_pool.view(dt).view(4, 90, BT, 2, dim) if layout == 0 else eng.hbm_pool.view(dt).view(90, 4, BT, 2, dim).transpose(0, 1),
              eng.tail_pool.view(dt).view(3, 4, BT, 2, dim).transpose(0, 1)]

    def keys(layer, kv):
        rows = [(caches[0], x) if x < 90 else (caches[1], x - 90) for x in table[0, :-(-kv // BT)].tolist()]
        return [torch.cat([c[2 * layer + y, x] for c, x in rows])[:kv].double() for y in (0, 1)]

    def step(position, kv, n, sparse):
        """n new tokens from `position` on; the sequence holds kv with them."""
        batch = (table, ints(0, n), ints(kv))
        for layer in range(2):
            q, k, v = (torch.empty(n, h, dim, dtype=dt, device="cuda").normal_(generator=g) for h in (hq, 2, 2))
            at = torch.arange(position, position + n, dtype=torch.int32, device="cuda")
            turned = eng.append_kv(layer, k, v, *batch, rope=rope, positions=at, q=q)
            eng.bound_keys(layer, bounds, *batch, n_tokens=n)
            kk, vv = keys(layer, kv)
            want_k, size = rotated(torch, k.double(), at[None].long(), freqs, [0] * (dim // 2), dim, False)
            assert bool(((kk[-n:] - want_k).abs() <= 2.0 ** -8 * want_k.abs() + 2.0 ** -20 * size).all())
            lse = torch.empty(n, hq, device="cuda")
            see = torch.arange(kv, device="cuda") <= torch.arange(kv - n, kv, device="cuda")[:, None]
            see = see[:, None].expand(n, hq, kv)
            if sparse:
                blocks = eng.select_blocks(layer, turned, bounds, *batch, 8)
                o = eng.attend_blocks(layer, turned, blocks, *batch, lse=lse)
                chosen = torch.zeros(n, 2, 72, dtype=torch.bool, device="cuda").scatter_(2, torch.where(blocks < 0, 71, blocks).long(), True)
                assert bool((chosen[:, :, :71].sum(2) == 8).all())
                see = see & chosen.repeat_interleave(BT, 2)[:, :, :kv].repeat_interleave(3, 1)
            else:
                o = eng.attend(layer, turned, *batch, lse=lse)
            x = torch.einsum("ihgd,jhd->ihgj", turned.double().view(n, 2, 3, dim), kk).reshape(n, hq, kv) * dim ** -0.5
            p = torch.softmax(torch.where(see, x, -math.inf), -1)
            want = torch.einsum("ihgj,jhd->ihgd", p.view(n, 2, 3, kv), vv).reshape(n, hq, dim)
            size = torch.einsum("ihgj,jhd->ihgd", p.view(n, 2, 3, kv), vv.abs()).reshape(n, hq, dim)
            assert bool(((o.double() - want).abs() <= 2.0 ** -8 * want.abs() + size * (2.0 ** -8 + 2.0 ** -10)).all())
            if not sparse:
                before = weights.clone()
                eng.weigh_blocks(layer, turned, lse, *batch, weights=weights, out=weights)
                new = torch.nn.functional.pad(p.sum((0, 1)), (0, 70 * BT - kv)).view(70, BT).sum(1)
                assert torch.allclose(weights[0].double(), before[0].double() + new, rtol=1e-4, atol=1e-6)
        eng.kv_check()

    step(0, 700, 700, False)
    step(700, 1000, 300, False)
    assert abs(float(weights.sum()) / (2 * 1000 * hq) - 1) < 1e-4
    for i in range(3):
        step(1000 + i, 1001 + i, 1, True)
    new_table, kv_len, new_weights, evicted = eng.evict_blocks(weights, table, ints(1003), 30, first=1, last=4)
    gone = evicted[0][evicted[0] >= 0].cpu().numpy()
    assert kv_len.tolist() == [1003 - 33 * BT] and len(gone) == 33 and bool((gone < 90).all())
    assert sorted([*gone, *new_table[0, :30].tolist()]) == sorted(table[0, :63].tolist())
    eng.prefill_done(0)
    eng.release(B.TIER_HBM, gone)
    assert eng.get_stats()["occ_hbm"] == 62 - 33
    table.copy_(new_table)
    weights.copy_(new_weights)
    kv = int(kv_len[0])
    for i in range(5):
        step(1003 + i, kv + 1 + i, 1, i % 2 == 0)
    assert (kv + 5) % BT == 0
    table[0, 30] = eng.n_hbm_blocks + 1         # that block is full: the next tail block
    step(1008, kv + 5 + 3, 3, True)
    eng.close()
