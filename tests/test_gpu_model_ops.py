"""append_kv and attend against their definitions in 64 bits. Unused parts of the pool hold NaN, so anything read that
should not be shows up; everything an operator must leave alone is compared bit by bit."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2609_39819_b200 import workloads as W

pytestmark = pytest.mark.gpu
BT = 16


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_39819_b200 import binding
    binding.load_library()
    return binding


class Setup:
    """An engine whose pool is NaN except for the tokens its sequences hold. new[s] tokens on top of past[s]."""

    def __init__(self, B, new, past, heads=2, group=2, dim=64, dtype="bf16", layout=0, layers=2, layer=1, seed=0, tail=False,
                 strided=False, pad=0, spare_blocks=2, q_gain=1.0):
        import torch
        self.torch, self.B = torch, B
        g = torch.Generator("cuda").manual_seed(1000 + seed)
        self.dt = dt = torch.bfloat16 if dtype == "bf16" else torch.float16
        self.u = torch.finfo(dt).eps / 2
        self.new, self.past, self.heads, self.group, self.dim, self.layer = new, past, heads, group, dim, layer
        self.kv = [max(0, n + p) for n, p in zip(new, past)]
        blocks = [-(-k // BT) for k in self.kv]
        n_all = sum(blocks) + 5
        n_tail = n_all // 2 if tail else 0
        n_slots = n_all - n_tail
        self.eng = eng = B.Engine(n_layers=layers, n_kv_heads=heads, head_dim=dim, pool_layout=layout, n_hbm_blocks=n_slots,
                                  n_host_blocks=0, max_contexts=2, max_messages=16, max_tokens=256, n_tail_blocks=n_tail)
        pool = eng.hbm_pool.view(dt)
        pool.fill_(math.nan)
        chunks = 2 * layers
        self.pools = [pool.view(chunks, n_slots, BT, heads, dim) if layout == 0 else
                      pool.view(n_slots, chunks, BT, heads, dim).transpose(0, 1)]
        if n_tail:
            eng.tail_pool.view(dt).fill_(math.nan)
            self.pools.append(eng.tail_pool.view(dt).view(n_tail, chunks, BT, heads, dim).transpose(0, 1))
        self.n_slots = n_slots
        perm = torch.randperm(n_all, generator=g, device="cuda").int().cpu()
        width = max(blocks + [1]) + spare_blocks
        self.host_table = torch.full((len(new), width), 0x7FFFFFF0, dtype=torch.int32)   # unused entries are no slots
        at = 0
        for i, b in enumerate(blocks):
            self.host_table[i, :b] = perm[at:at + b]
            at += b
        self.table = self.host_table.cuda()
        start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.q_start = torch.from_numpy(start).cuda()
        self.kv_len = torch.tensor(self.kv, dtype=torch.int32).cuda()
        t = self.t = int(start[-1])
        rows = t + pad
        self.rows = rows

        def tensor(h):
            if strided:     # heads of a fused projection, an odd distance apart
                x = torch.empty(rows, h * 3, dim + 5, dtype=dt, device="cuda").normal_(generator=g)
                return x[:, ::3, 2:2 + dim]
            return torch.empty(rows, h, dim, dtype=dt, device="cuda").normal_(generator=g)

        self.q, self.k, self.v = tensor(heads * group).mul_(q_gain), tensor(heads), tensor(heads)
        for i in range(len(new)):      # what the sequences held before
            for s, o, n in self._places(i, 0, max(0, self.kv[i] - new[i])):
                for c in (0, 1):
                    self._chunk(s, c)[o:o + n] = torch.empty(n, heads, dim, dtype=dt, device="cuda").normal_(generator=g)

    def _places(self, i, a, z):
        """(slot, offset, count) of tokens a .. z-1 of sequence i."""
        while a < z:
            n = min(BT - a % BT, z - a)
            yield int(self.host_table[i, a // BT]), a % BT, n
            a += n

    def _chunk(self, slot, c):
        pool, s = (self.pools[0], slot) if slot < self.n_slots else (self.pools[1], slot - self.n_slots)
        return pool[2 * self.layer + c, s]

    def put(self):
        """The new keys and values, unrotated, straight into the pool (for tests of attend alone)."""
        t0 = 0
        for n, kv, i in zip(self.new, self.kv, range(len(self.new))):
            at = max(kv - n, 0)
            for s, o, m in self._places(i, at, kv):
                row = t0 + at - (kv - n)
                self._chunk(s, 0)[o:o + m] = self.k[row:row + m]
                self._chunk(s, 1)[o:o + m] = self.v[row:row + m]
                at += m
            t0 += n

    def gather(self, i):
        """K and V of sequence i, [kv, heads, dim] in 64 bits."""
        torch = self.torch
        out = []
        for c in (0, 1):
            parts = [self._chunk(s, c)[o:o + n] for s, o, n in self._places(i, 0, self.kv[i])]
            out.append(torch.cat(parts).double() if parts else torch.zeros(0, self.heads, self.dim, dtype=torch.float64, device="cuda"))
        return out

    def reference(self, window=0, causal=True, scale=None):
        """out, lse and how far each may be off, in 64 bits."""
        torch = self.torch
        scale = self.dim ** -0.5 if scale is None else scale
        hq = self.heads * self.group
        out = torch.zeros(self.t, hq, self.dim, dtype=torch.float64, device="cuda")
        lse = torch.full((self.t, hq), -math.inf, dtype=torch.float64, device="cuda")
        tol, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
        t0, e32 = 0, 2.0 ** -24
        for i, n in enumerate(self.new):
            k, v = self.gather(i)
            kv = self.kv[i]
            own = torch.arange(n, device="cuda")[:, None] + (kv - n)
            key = torch.arange(kv, device="cuda")[None]
            see = (key <= own) if causal else torch.ones(n, kv, dtype=torch.bool, device="cuda")
            if window:
                see &= own - key < window
            some = see.any(1) if kv else torch.zeros(n, dtype=torch.bool, device="cuda")
            if kv and bool(some.any()):
                for h in range(hq):
                    q = self.q[t0:t0 + n, h].double()
                    kh, vh = k[:, h // self.group], v[:, h // self.group]
                    s = torch.where(see, q @ kh.T * scale, -math.inf)[some]
                    big = torch.where(see, q.abs() @ kh.abs().T * abs(scale), 0.0)[some].amax(1, keepdim=True)
                    L = torch.logsumexp(s, 1, keepdim=True)
                    p = torch.exp(s - L)
                    idx = t0 + torch.nonzero(some)[:, 0]
                    o = p @ vh
                    out[idx, h], lse[idx, h] = o, L[:, 0]
                    # scores: dim products summed in 32 bits and the scaling; sums over the keys in 32 bits; the powers and
                    # the final product a few units more; each probability and the result rounded once to the element type
                    ds = (self.dim + 4) * e32 * big
                    sums = (kv + 64) * e32
                    a = p @ vh.abs()
                    tol[idx, h] = self.u * o.abs() + a * (self.u + 2 * ds + 2 * sums) * (1 + self.u)
                    if self.dt == torch.float16:   # probabilities below 2^-14 and outputs below it have a fixed step of 2^-24
                        tol[idx, h] += 2.0 ** -25 * (1 + vh.abs().sum(0) / torch.exp(L - s.amax(1, keepdim=True)))
                    tol_l[idx, h] = (ds + sums)[:, 0] + 4 * e32 * L[:, 0].abs()
            t0 += n
        return out, lse, tol, tol_l

    def widened(self):
        """The block table with rows that could hold 320 K tokens more: the kernel for prompts is taken for fewer of them."""
        w = self.torch.full((self.table.shape[0], self.table.shape[1] + 20000), 0x7FFFFFF0, dtype=self.torch.int32, device="cuda")
        w[:, :self.table.shape[1]] = self.table
        return w

    def bits(self):
        return [p.clone().contiguous().view(self.torch.int16) for p in self.pools]


def check_attend(s, window=0, causal=True, scale=None, want_lse=True):
    """The result must not depend on what the kernel is chosen by: the hint, and how much a table row could hold."""
    torch = s.torch
    wide = s.widened()
    check_one(s, s.table, max(s.new), window, causal, scale, want_lse)
    check_one(s, wide, None, window, causal, scale, want_lse)       # many rows: the kernel for prompts
    check_one(s, s.table, 1, window, causal, scale, want_lse)       # the kernel for few rows
    check_one(s, wide, 1, window, causal, scale, want_lse)


def check_one(s, table, max_q_len, window, causal, scale, want_lse):
    torch = s.torch
    hq = s.heads * s.group
    guard = 7.25
    out = torch.full((s.rows, hq * 2, s.dim + 3), guard, dtype=s.dt, device="cuda")
    view = out[:, ::2, 1:1 + s.dim] if s.rows % 2 else out[:, :hq, :s.dim]
    lse = torch.full((s.rows, hq), guard, device="cuda") if want_lse else None
    before = s.bits()
    s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len, max_q_len=max_q_len, window=window, causal=causal, scale=scale,
                 out=view, lse=lse)
    s.eng.kv_check()
    want, wl, tol, tl = s.reference(window, causal, scale)
    got = view[:s.t].double()
    assert bool(torch.isfinite(got).all())
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), float(((got - want).abs() / (tol + 1e-30)).max()), torch.nonzero(bad)[:4].tolist())
    if want_lse:
        g = lse[:s.t].double()
        none = torch.isinf(wl)
        assert bool((g[none] == -math.inf).all())
        assert not bool(((g - wl).abs() > tl)[~none].any()), float((g - wl).abs()[~none].max())
        assert bool((lse[s.t:] == guard).all())
    # rows behind the last sequence, and everything between the rows, stay
    mask = torch.ones_like(out, dtype=torch.bool)
    (mask[:, ::2, 1:1 + s.dim] if s.rows % 2 else mask[:, :hq, :s.dim])[:s.t] = False
    assert bool((out[mask] == guard).all())
    for a, b in zip(before, s.bits()):
        assert torch.equal(a, b)       # the pool is only read
    return view


# sequences: (new, past) each; the shapes of decode steps, prompts, chunks, empty and odd ones
STEP = ([1] * 6, [0, 1, 15, 16, 300, 1000])
RAGGED = ([5, 0, 33, 1, 130], [0, 40, 7, 511, 255])
PROMPT = ([300], [0])
CHUNK = ([70, 3], [700, 2500])
EMPTY_ROWS = ([6, 4, 40, 1], [-4, -4, -20, 0])      # kv_len below the number of new tokens: leading rows see nothing
BATCHES = {"step": STEP, "ragged": RAGGED, "prompt": PROMPT, "chunk": CHUNK, "empty": EMPTY_ROWS}


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("dtype,layout,heads,group,dim", [("bf16", 0, 2, 4, 128), ("fp16", 1, 2, 1, 64), ("bf16", 1, 1, 7, 64),
                                                           ("fp16", 0, 2, 12, 128), ("bf16", 0, 3, 2, 80), ("fp16", 1, 1, 3, 256)])
def test_attend_shapes(B, batch, dtype, layout, heads, group, dim):
    s = Setup(B, *BATCHES[batch], heads=heads, group=group, dim=dim, dtype=dtype, layout=layout, seed=len(batch) + dim, q_gain=2.0)
    s.put()
    check_attend(s)


@pytest.mark.parametrize("dim", [64, 128, 32])
@pytest.mark.parametrize("batch", ["step", "ragged", "chunk", "empty"])
@pytest.mark.parametrize("window", [1, 16, 100, 5000])
def test_attend_window(B, batch, window, dim):
    s = Setup(B, *BATCHES[batch], heads=2, group=3, dim=dim, seed=window)
    s.put()
    check_attend(s, window=window)
    # blocks that no query of a sequence sees need no valid slot
    for i, (n, kv) in enumerate(zip(s.new, s.kv)):
        first = max(0, kv - n + 1 - window) if n else kv
        s.host_table[i, :first // BT] = -1
    s.table.copy_(s.host_table)
    got = s.torch.empty(s.t, 6, dim, dtype=s.dt, device="cuda")
    s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len, window=window, out=got)
    s.eng.kv_check()
    assert bool(s.torch.isfinite(got).all())


@pytest.mark.parametrize("dim", [64, 128, 96])
@pytest.mark.parametrize("batch", BATCHES)
def test_attend_full(B, batch, dim):
    s = Setup(B, *BATCHES[batch], heads=2, group=2, dim=dim, dtype="fp16", seed=3)
    s.put()
    check_attend(s, causal=False)
    check_attend(s, causal=False, scale=0.01, want_lse=False)


@pytest.mark.parametrize("dim,group", [(64, 5), (128, 4), (24, 2)])
@pytest.mark.parametrize("batch", ["step", "ragged", "chunk"])
def test_attend_strides_tail_blocks_and_padding(B, batch, dim, group):
    s = Setup(B, *BATCHES[batch], heads=2, group=group, dim=dim, strided=True, tail=True, pad=9, seed=4)
    s.put()
    check_attend(s)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 2, 3, 8, 9, 17, 31, 32, 33, 63, 64, 65, 127, 129])
def test_attend_every_chunk_size(B, dim, new):
    s = Setup(B, [new, new], [0, 1500 + new], heads=1, group=4, dim=dim, seed=new)
    s.put()
    check_attend(s)


@pytest.mark.parametrize("dim,new,past,heads,group", [(128, 1, 70000, 1, 8), (64, 1, 90001, 2, 2), (128, 40, 40000, 1, 4),
                                                       (64, 200, 20011, 1, 1), (128, 1, 5000, 1, 16), (128, 1, 5000, 1, 40)])
def test_attend_long(B, dim, new, past, heads, group):
    s = Setup(B, [new], [past], heads=heads, group=group, dim=dim, layers=1, layer=0, q_gain=3.0, seed=past)
    s.put()
    check_attend(s)


@pytest.mark.parametrize("past", [[80000], [30011, 50000, 100, 0]])
def test_attend_work_that_ctas_take_over(B, past):
    """Enough blocks that part of the work is left to the CTAs that are through first; who takes what must not show."""
    import torch
    s = Setup(B, [1] * len(past), past, heads=8, group=2, dim=64, layers=1, layer=0, q_gain=2.0, seed=77)
    s.put()
    check_attend(s)
    first = s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len)
    for _ in range(10):
        assert torch.equal(first, s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len))


def test_attend_many_sequences(B):
    rng = np.random.default_rng(5)
    n = 700
    s = Setup(B, [int(x) for x in rng.integers(0, 3, n)], [int(x) for x in rng.integers(0, 60, n)], heads=1, group=2, dim=64, seed=6)
    s.put()
    check_attend(s)


@pytest.mark.parametrize("n,new,past", [(40, 90, 3000), (540, 40, 260), (3, 700, 9000)])
def test_attend_ragged_sequences_in_pieces(B, n, new, past):
    """Pieces of one length over sequences of many, more sequences than are ordered (or weighed) at a time, some with nothing."""
    rng = np.random.default_rng(n)
    news = [int(x) for x in rng.integers(0, new, n)]
    s = Setup(B, news, [int(x) for x in rng.integers(0, past, n)], heads=1, group=3, dim=64 if n > 500 else 128, seed=n)
    s.put()
    check_attend(s)


def test_attend_scratch_at_any_16_bytes(B):
    """Partial results in scratch that is aligned to 16 bytes and no more, with something else before it."""
    import torch
    s = Setup(B, [300], [4000], heads=2, group=2, dim=128, seed=5)
    s.put()
    want = s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len)
    real = torch.empty
    offset = []

    def empty(*size, **kw):
        if kw.get("dtype") is torch.uint8 and len(size) == 1 and isinstance(size[0], int):
            offset.append(size[0])
            return real(size[0] + 16, **kw)[16:]
        return real(*size, **kw)

    s.eng._attend_native = lambda *args: NotImplemented          # the marshalling in Python allocates with torch.empty
    torch.empty = empty
    try:
        got = s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len)
    finally:
        torch.empty = real
    assert offset and torch.equal(want, got)


@pytest.mark.parametrize("axes,inter", [(1, False), (3, True)])
def test_native_and_python_marshalling_make_the_same_call(B, axes, inter):
    import torch
    s = Setup(B, [3, 0, 70], [200, 0, 9], heads=2, group=3, dim=64, seed=4)
    rope = B.Rope(64, sections=[10, 10, 12] if axes > 1 else None, interleaved=inter)
    pos = torch.arange(axes * s.rows, dtype=torch.int32, device="cuda").view(axes, s.rows)[:, :s.rows] * 3
    args = (s.table, s.q_start, s.kv_len)
    lse = torch.empty(2, s.rows, 6, device="cuda").fill_(1.0)
    got = []
    for i in range(2):
        if i:
            for name in ("_append_native", "_attend_native"):
                assert callable(getattr(s.eng, name))
                setattr(s.eng, name, lambda *a: NotImplemented)
        for p in s.pools:
            p.zero_()
        q = torch.zeros_like(s.q)
        r = s.eng.append_kv(s.layer, s.k, s.v, *args, rope=rope, positions=pos, q=s.q, q_out=q)
        assert r is q
        assert s.eng.append_kv(s.layer, s.k, s.v, *args, rope=rope, positions=pos) is None
        out = torch.zeros_like(s.q)
        assert s.eng.attend(s.layer, q, *args, window=50, scale=0.2, max_q_len=70, out=out, lse=lse[i]) is out
        new = s.eng.attend(s.layer, q, *args, causal=False)
        s.eng.kv_check()
        got.append([q, out, new[:s.t].clone(), lse[i]] + s.bits())
    for x, y in zip(*got):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,layout", [("bf16", 0), ("fp16", 1)])
@pytest.mark.parametrize("dim", [1, 7, 8, 33, 63, 65, 80, 96, 120, 127, 129, 160, 192, 250, 256])
def test_attend_every_head_size(B, dim, dtype, layout):
    """Heads that fill a part of a tile's columns, that 16-byte copies reach or do not; one part of the keys or several."""
    s = Setup(B, [1, 37, 0, 3], [700, 20, 5, 4000], dtype=dtype, layout=layout, heads=2, group=3, dim=dim, seed=dim)
    s.put()
    check_attend(s, window=300 if dim % 2 else 0)
    s = Setup(B, [300, 1], [40, 0], dtype=dtype, layout=layout, heads=1, group=2, dim=dim, seed=dim)
    s.put()
    check_attend(s)


def test_attend_scores_that_climb_and_scores_of_one_huge_key(B):
    """The running maximum has to be raised again and again, by little and by much, in either kernel."""
    import torch
    for new in (1, 100):
        s = Setup(B, [new], [3000], heads=1, group=2, dim=128, dtype="bf16", seed=8)
        s.q.copy_(s.q.abs())
        s.put()
        for slot, o, n in s._places(0, 0, s.kv[0]):
            at = [b for b in range(s.host_table.shape[1]) if int(s.host_table[0, b]) == slot][0] * BT + o
            ramp = torch.arange(at, at + n, device="cuda")[:, None, None] / s.kv[0]
            c = s._chunk(slot, 0)[o:o + n]
            c.copy_(ramp.expand_as(c) * 0.9 + 0.02 * c.float())
        s._chunk(int(s.host_table[0, 100]), 0)[3] = 3.0
        check_attend(s)


@pytest.mark.parametrize("dim", [64, 128, 72])
@pytest.mark.parametrize("new", [1, 40, 200])
def test_a_nan_or_an_overflow_stays_with_the_rows_that_see_it(B, new, dim):
    """A NaN in a query spoils its row, a NaN in a key or a score beyond the range the rows that see the key; nobody else."""
    import torch
    for key_back in (0, 3, 6, 7, 29, 120):          # how far before the end the bad key lies: every way a power is made
        for bad in (math.nan, math.inf):
            s = Setup(B, [new, 5], [300, 40], heads=2, group=2, dim=dim, dtype="bf16", seed=9)
            s.q[:, :, 0] = s.q[:, :, 0].abs() + 0.5
            s.put()
            at = s.kv[0] - 1 - key_back
            s._chunk(int(s.host_table[0, at // BT]), 0)[at % BT, 1, 0] = bad
            s.q[new - 1, 0, 3] = math.nan
            want_bad = torch.zeros(s.t, 4, dtype=torch.bool, device="cuda")
            own = torch.arange(new, device="cuda") + 300
            want_bad[:new, 2:] = (own >= at)[:, None]
            want_bad[new - 1, 0] = True
            for table in (s.table, s.widened()):
                got = s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len)
                s.eng.kv_check()
                assert torch.equal(torch.isnan(got).all(-1), want_bad), (key_back, bad)
                assert torch.equal(torch.isfinite(got).all(-1), ~want_bad), (key_back, bad)


# ---- append -----------------------------------------------------------------------------------------------
def rotated(torch, x, pos, freqs, axis, rot, interleaved):
    """x: [tokens, heads, dim] in 64 bits, pos: [axes, tokens]. Also the size the rounding errors scale with."""
    y, size = x.clone(), x.abs()
    for j in range(rot // 2):
        a = pos[axis[j]].double() * freqs[j]
        u, w = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
        y[..., u], y[..., w] = x[..., u] * c - x[..., w] * s, x[..., w] * c + x[..., u] * s
        size[..., u] = size[..., w] = x[..., u].abs() + x[..., w].abs()
    return y, size


@pytest.mark.parametrize("batch", ["step", "ragged", "prompt", "empty"])
@pytest.mark.parametrize("dtype,layout,heads,group,dim,rot,inter,axes,strided",
                         [("bf16", 0, 2, 4, 128, 128, False, 1, False), ("fp16", 1, 2, 3, 64, 64, True, 1, False),
                          ("bf16", 1, 1, 7, 64, 32, False, 3, False), ("fp16", 0, 3, 2, 128, 64, True, 3, True),
                          ("bf16", 0, 2, 1, 80, 40, False, 1, False), ("fp16", 0, 2, 2, 64, 64, False, 1, True),
                          ("bf16", 1, 1, 1, 48, 6, True, 2, False), ("bf16", 0, 2, 2, 64, 0, False, 1, False)])
def test_append(B, batch, dtype, layout, heads, group, dim, rot, inter, axes, strided):
    import torch
    s = Setup(B, *BATCHES[batch], heads=heads, group=group, dim=dim, dtype=dtype, layout=layout, strided=strided, tail=dim == 64,
              pad=5, seed=11)
    freqs = [50000.0 ** (-2 * j / max(rot, 1)) for j in range(rot // 2)]
    axis = [j % axes for j in range(rot // 2)]
    rope = B.Rope(rot, theta=50000.0, axis_of=axis if axes > 1 else None, interleaved=inter)
    pos = torch.randint(-50, 300000, (axes, s.rows), device="cuda", dtype=torch.int32) if axes > 1 else None
    seq = np.repeat(np.arange(len(s.new)), s.new)
    first = np.concatenate([[0], np.cumsum(s.new)])
    index = np.array([s.kv[i] - s.new[i] + t - first[i] for t, i in enumerate(seq)], dtype=np.int64)
    p64 = pos[:, :s.t] if axes > 1 else torch.from_numpy(index).cuda()[None]
    before = s.bits()
    q_out = torch.full((s.rows, heads * group, dim + (3 if strided else 0)), 7.25, dtype=s.dt, device="cuda")[..., :dim]
    got_q = s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope, positions=pos, q=s.q, q_out=q_out)
    short = any(kv < n for kv, n in zip(s.kv, s.new))
    if short:        # tokens in front of their sequence's first place: reported, not written
        with pytest.raises(B.KvtError) as exc:
            s.eng.kv_check()
        assert exc.value.code == B.E_RANGE
    else:
        s.eng.kv_check()
    assert got_q is q_out and bool((q_out[s.t:] == 7.25).all())
    keep = torch.from_numpy(index >= 0).cuda()
    for x, is_q in ((s.q, True), (s.k, False)):
        want, size = rotated(torch, x[:s.t].double(), p64, freqs, axis, rot, inter)
        if is_q:
            got = q_out[:s.t].double()
        else:
            got = torch.stack([s._chunk(int(s.host_table[i, t // BT]), 0)[t % BT] if t >= 0 else s.k[j]
                               for j, (i, t) in enumerate(zip(seq, index))]).double() if s.t else want
        # the angle is exact to 1e-10 in 64 bits and its turn is rounded once to 32 bits (2^-25 of a turn, 2 pi 2^-25
        # radians), sine and cosine to an ulp or two, the rotation to 3 roundings; then one rounding to the element type
        tol = s.u * want.abs() + size * (2 * math.pi * 2.0 ** -25 + 8 * 2.0 ** -24) * (1 + s.u)
        if dtype == "fp16":
            tol = tol + 2.0 ** -25
        bad = ((got - want).abs() > tol)[keep]
        assert not bool(bad.any()), (is_q, int(bad.sum()))
        tail = slice(rot, dim)
        assert torch.equal(got[..., tail][keep], x[:s.t].double()[..., tail][keep])
    for j, (i, t) in enumerate(zip(seq, index)):
        if t >= 0:
            slot = int(s.host_table[i, t // BT])
            assert torch.equal(s._chunk(slot, 1)[t % BT], s.v[j])
            for c in (0, 1):      # put back what was there, so that the rest compares
                pool = 0 if slot < s.n_slots else 1
                s._chunk(slot, c)[t % BT] = before[pool].view(s.dt)[2 * s.layer + c, slot - (s.n_slots if pool else 0), t % BT]
    for a, b in zip(before, s.bits()):
        assert torch.equal(a, b)


def test_append_in_place_and_without_queries_or_rotation(B):
    import torch
    s = Setup(B, [20, 3], [5, 100], heads=2, group=4, dim=128, seed=21)
    rope = B.Rope(128)
    want = s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope, q=s.q)
    pool = s.bits()
    q = s.q.clone()
    assert s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope, q=q, q_out=q) is q
    assert torch.equal(q, want)
    assert s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope) is None
    assert all(torch.equal(a, b) for a, b in zip(pool, s.bits()))
    s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len)
    k, v = s.gather(1)
    assert torch.equal(k[100:], s.k[20:].double()) and torch.equal(v[100:], s.v[20:].double())
    s.eng.kv_check()


def test_rope_frequencies_of_the_callers_own(B):
    import torch
    s = Setup(B, [40], [0], heads=1, group=1, dim=64, dtype="fp16", seed=22)
    f = [0.5 / (j + 1) for j in range(16)]
    got = s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=B.Rope(32, freqs=f), q=s.q)
    want, _ = rotated(torch, s.q.double(), torch.arange(40, device="cuda")[None], f, [0] * 16, 32, False)
    assert float((got.double() - want).abs().max()) < 2.0 ** -9      # values below 8: half a step is 2^-9 at most
    secs = B.Rope(32, sections=[4, 6, 6])
    assert secs.n_axes == 3 and secs.axis_of.tolist() == [0] * 4 + [1] * 6 + [2] * 6


# ---- refusals and reports -----------------------------------------------------------------------------------
def test_refusals(B):
    import torch
    s = Setup(B, [4, 4], [10, 20], heads=2, group=2, dim=64, seed=31)
    e, L = s.eng, s.layer
    good = (s.table, s.q_start, s.kv_len)

    def refused(kind, f):
        with pytest.raises(kind):
            f()

    refused(B.KvtError, lambda: e.attend(2, s.q, *good))                                   # layer
    refused(B.KvtError, lambda: e.attend(L, s.q[:, :3], *good))                            # heads do not divide
    refused(B.KvtError, lambda: e.attend(L, s.q, *good, window=4, causal=False))
    refused(B.KvtError, lambda: e.attend(L, s.q, *good, scale=-1.0))
    refused(B.KvtError, lambda: e.attend(L, s.q, *good, scale=math.nan))
    refused(ValueError, lambda: e.attend(L, s.q.float(), *good))
    refused(ValueError, lambda: e.attend(-1, s.q, *good))
    refused(ValueError, lambda: e.attend(L, s.q, *good, window=-4))
    refused(ValueError, lambda: e.append_kv(-1, s.k, s.v, *good))
    refused(ValueError, lambda: e.attend(L, s.q, *good, out=s.q[:, :1].expand(-1, 4, -1)))
    refused(ValueError, lambda: e.attend(L, s.q[..., :32], *good))
    refused(ValueError, lambda: e.attend(L, s.q.transpose(1, 2), *good))
    refused(ValueError, lambda: e.attend(L, s.q.cpu(), *good))
    refused(ValueError, lambda: e.attend(L, s.q, s.table.long(), s.q_start, s.kv_len))
    refused(ValueError, lambda: e.attend(L, s.q, s.table, s.q_start[:2], s.kv_len))
    refused(ValueError, lambda: e.attend(L, s.q, s.table.cpu(), s.q_start, s.kv_len))
    refused(ValueError, lambda: e.attend(L, s.q, *good, lse=torch.empty(8, 2, device="cuda")))
    refused(ValueError, lambda: e.attend(L, s.q, *good, out=torch.empty(8, 4, 64, device="cuda")))
    refused(ValueError, lambda: e.append_kv(L, s.k, s.v.half(), *good))
    refused(ValueError, lambda: e.append_kv(L, s.k, s.v[:3], *good))
    refused(ValueError, lambda: e.append_kv(L, s.k, s.v, *good, q_out=s.q))
    refused(ValueError, lambda: e.append_kv(L, s.k, s.v, *good, positions=torch.zeros(8, dtype=torch.int32, device="cuda")))
    refused(ValueError, lambda: e.append_kv(L, s.k, s.v, *good, rope=B.Rope(64, sections=[8, 12, 12])))
    refused(ValueError, lambda: e.append_kv(L, s.k, s.v, *good, rope=B.Rope(64, sections=[8, 12, 12]),
                                            positions=torch.zeros(2, 8, dtype=torch.int32, device="cuda")))
    refused(B.KvtError, lambda: e.append_kv(L, s.k, s.v, *good, rope=B.Rope(66)))          # more than a head
    refused(ValueError, lambda: e.set_tail_pool(torch.empty(8, device="cuda")))
    e.kv_check()
    meta = B.Engine(n_layers=2, n_kv_heads=2, head_dim=64, n_hbm_blocks=8, n_host_blocks=0, metadata_only=True, max_tokens=256)
    refused(B.KvtError, lambda: meta.attend(0, s.q, *good))
    refused(B.KvtError, lambda: meta.append_kv(0, s.k, s.v, *good))
    wide = B.Engine(n_layers=2, n_kv_heads=2, head_dim=64, elem_bytes=4, n_hbm_blocks=8, n_host_blocks=0, max_tokens=256)
    refused(B.KvtError, lambda: wide.attend(0, s.q, *good))
    deep = B.Engine(n_layers=1, n_kv_heads=1, head_dim=264, n_hbm_blocks=8, n_host_blocks=0, max_tokens=256)
    refused(B.KvtError, lambda: deep.attend(0, torch.empty(8, 1, 264, dtype=torch.bfloat16, device="cuda"), *good))
    # through the C ABI: scratch too small, NULL tensors, misaligned addresses
    a = B.AttendArgs(B.Batch(2, 8, s.table.shape[1], 0, s.table.stride(0), s.q_start.data_ptr(), s.kv_len.data_ptr(),
                             s.table.data_ptr()), L, 0, 4, 0, 0, 0.0, s.q.data_ptr(), s.q.data_ptr(), None, 256, 64, 256, 64)
    lib = e.L
    for field, value in (("q", None), ("out", None), ("q", a.q + 1), ("lse", a.q + 2), ("flags", 2), ("dtype", 2), ("n_q_heads", 0)):
        old = getattr(a, field)
        setattr(a, field, value)
        assert lib.kvt_attend(e.h, C.byref(a), None) == B.E_INVAL, field
        setattr(a, field, old)
    need = lib.kvt_attend_scratch_bytes(e.h, C.byref(a))
    if need:
        assert lib.kvt_attend(e.h, C.byref(a), None) == B.E_BUFSZ
    torch.cuda.synchronize()


@pytest.mark.parametrize("dim", [64, 128, 40])
@pytest.mark.parametrize("new,wide", [(1, False), (50, False), (50, True)])
def test_bad_slots_and_lengths_are_reported_and_harmless(B, dim, new, wide):
    import torch
    s = Setup(B, [new, new], [100, 200], heads=2, group=4, dim=dim, tail=True, seed=41)
    s.put()
    if wide:
        s.table = s.widened()
    sound = s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len)
    s.eng.kv_check()

    def report(f):
        r = f()
        with pytest.raises(B.KvtError) as exc:
            s.eng.kv_check()
        assert exc.value.code == B.E_RANGE
        s.eng.kv_check()          # cleared
        return r

    n_all = s.n_slots + s.pools[1].shape[1]
    for bad in (n_all, -1, 0x7FFFFFFF):
        t = s.table.clone()
        t[1, 3] = bad
        got = report(lambda: s.eng.attend(s.layer, s.q, t, s.q_start, s.kv_len))
        assert bool(torch.isfinite(got).all()) and torch.equal(got[:new], sound[:new])
        before = s.bits()
        t = s.table.clone()
        t[1, (s.kv[1] - 1) // BT] = bad
        report(lambda: s.eng.append_kv(s.layer, s.k, s.v, t, s.q_start, s.kv_len))
        s.put()
        assert all(torch.equal(a, b) for a, b in zip(before, s.bits()))
    # lengths beyond the table row, starts that decrease or pass the rows
    report(lambda: s.eng.attend(s.layer, s.q, s.table[:, :5], s.q_start, s.kv_len))
    report(lambda: s.eng.attend(s.layer, s.q, s.table, s.q_start + torch.tensor([0, 0, 7], dtype=torch.int32, device="cuda"), s.kv_len))
    report(lambda: s.eng.attend(s.layer, s.q, s.table, s.q_start.flip(0).contiguous(), s.kv_len))
    report(lambda: s.eng.append_kv(s.layer, s.k, s.v, s.table[:, :5], s.q_start, s.kv_len))
    report(lambda: s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start + torch.tensor([0, 0, 7], dtype=torch.int32, device="cuda"), s.kv_len))
    # the same tokens in every other of 400 sequences: reported, and over at once
    up_down = torch.tensor([0, s.t] * 200 + [0], dtype=torch.int32, device="cuda")
    many = s.table[:1].expand(400, -1).contiguous()
    report(lambda: s.eng.attend(s.layer, s.q, many, up_down, s.kv_len[:1].expand(400).contiguous()))
    report(lambda: s.eng.append_kv(s.layer, s.k, s.v, many, up_down, s.kv_len[:1].expand(400).contiguous()))
    rope = B.Rope(dim, axis_of=[j % 3 for j in range(dim // 2)])
    rope.n_axes = 2
    report(lambda: s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope,
                                   positions=torch.zeros(2, s.t, dtype=torch.int32, device="cuda")))


def test_nothing_to_do(B):
    import torch
    s = Setup(B, [0, 0], [10, 20], heads=2, group=2, dim=64, seed=51)
    assert s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len).shape == (0, 4, 64)
    s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len)
    empty = torch.zeros(0, 3, dtype=torch.int32, device="cuda")
    s.eng.attend(s.layer, s.q, empty, s.q_start[:1], s.kv_len[:0])
    # no sequence has a token, the rows are padding
    out = torch.full((5, 4, 64), 3.0, dtype=s.dt, device="cuda")
    s.eng.attend(s.layer, torch.zeros_like(out), s.table, s.q_start, s.kv_len, out=out)
    s.eng.append_kv(s.layer, out[:, :2], out[:, :2], s.table, s.q_start, s.kv_len)
    s.eng.kv_check()
    assert bool((out == 3.0).all())


# ---- streams, graphs, the set as it is used --------------------------------------------------------------------
@pytest.mark.parametrize("new,wide", [(1, False), (1, True), (60, False), (60, True)])
def test_captured_and_replayed_with_other_lengths(B, new, wide):
    """Two graphs of the same engine, replayed at once on two streams, with lengths changed after the capture."""
    import torch
    s = Setup(B, [new] * 3, [900, 40, 2000], heads=2, group=4, dim=128, seed=61)
    s.put()
    if wide:
        s.table = s.widened()
    rope = B.Rope(128)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    kv = [s.kv_len.clone(), s.kv_len.clone()]
    graphs, outs = [], []
    s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len)       # first use outside a capture
    torch.cuda.synchronize()
    for st, k in zip(streams, kv):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            outs.append(s.eng.attend(s.layer, s.q, s.table, s.q_start, k, max_q_len=new))
        graphs.append(g)
    for shift in (0, 17, 350):
        for i, k in enumerate(kv):
            k.copy_(s.kv_len - shift * i)
            k.clamp_(min=0)
        torch.cuda.synchronize()
        for _ in range(20):
            for st, g in zip(streams, graphs):
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for i, k in enumerate(kv):
            want = s.eng.attend(s.layer, s.q, s.table, s.q_start, k, max_q_len=new)
            assert torch.equal(outs[i], want)
    s.eng.kv_check()
    g = torch.cuda.CUDAGraph()
    before = s.bits()
    with torch.cuda.graph(g):
        q = s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope, q=s.q)
    assert all(torch.equal(a, b) for a, b in zip(before, s.bits()))
    g.replay()
    got, pool = q.clone(), s.bits()
    assert torch.equal(s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=rope, q=s.q), got)
    assert all(torch.equal(a, b) for a, b in zip(pool, s.bits()))
    s.eng.kv_check()


def test_same_call_gives_the_same_bits(B):
    import torch
    for new, past in (([1] * 20, list(range(0, 6000, 300))), ([90, 300], [3000, 20])):
        s = Setup(B, new, past, heads=2, group=4, dim=128, seed=71)
        s.put()
        for table in (s.table, s.widened()):
            first = s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len)
            for _ in range(5):
                assert torch.equal(first, s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len))


@pytest.mark.parametrize("layout", [0, 1])
def test_session_from_tokens_to_attention_through_eviction(B, layout):
    """The set as it is used: a context's blocks are admitted, its prompt is appended and attended to chunk by chunk,
    its blocks are pushed to the host tier and come back into other slots, and the next turn attends over them."""
    import torch
    geo = W.Geometry("small", 2, 2, 64)
    eng = B.Engine(n_hbm_blocks=40, n_host_blocks=64, max_contexts=4, max_messages=64, max_tokens=4096, pool_layout=layout,
                   n_tail_blocks=4, **geo.kwargs())
    g = torch.Generator("cuda").manual_seed(1)
    dt, hq, scale = torch.bfloat16, 6, 64 ** -0.5
    rope = B.Rope(64)
    tokens = np.arange(900, dtype=np.uint32)
    ks = torch.empty(2, 900, 2, 64, dtype=dt, device="cuda").normal_(generator=g)      # per layer, by token index
    vs = torch.empty(2, 900, 2, 64, dtype=dt, device="cuda").normal_(generator=g)
    qs = torch.empty(2, 900, hq, 64, dtype=dt, device="cuda").normal_(generator=g)

    def table_of(ctx, total):
        keys, tier, slot = eng.get_block_map(ctx)
        assert bool((tier == B.TIER_HBM).all())
        t = torch.full((1, 60), -1, dtype=torch.int32)
        t[0, :len(slot)] = torch.from_numpy(slot.astype(np.int32))
        if total % BT:
            t[0, len(slot)] = eng.n_hbm_blocks + 2          # the partly filled block lies in a tail block
        return t.cuda()

    def chunk(ctx, a, z):
        table = table_of(ctx, z)
        args = (table, torch.tensor([0, z - a], dtype=torch.int32).cuda(), torch.tensor([z], dtype=torch.int32).cuda())
        for layer in range(2):
            q = eng.append_kv(layer, ks[layer, a:z], vs[layer, a:z], *args, rope=rope, q=qs[layer, a:z])
            o = eng.attend(layer, q, *args, max_q_len=z - a)
            eng.kv_check()
            pos = torch.arange(z, device="cuda")[None]
            freqs = [10000.0 ** (-2 * j / 64) for j in range(32)]
            kk, _ = rotated(torch, ks[layer, :z].double(), pos, freqs, [0] * 32, 64, False)
            qq, _ = rotated(torch, qs[layer, a:z].double(), pos[:, a:], freqs, [0] * 32, 64, False)
            x = torch.einsum("ihgd,jhd->hgij", qq.view(z - a, 2, 3, 64), kk) * scale
            x = x.masked_fill(torch.arange(z, device="cuda")[None] > torch.arange(a, z, device="cuda")[:, None], -math.inf)
            p = torch.softmax(x, -1)
            want = torch.einsum("hgij,jhd->ihgd", p, vs[layer, :z].double()).reshape(z - a, hq, 64)
            size = torch.einsum("hgij,jhd->ihgd", p, vs[layer, :z].double().abs()).reshape(z - a, hq, 64)
            # q and k are rounded after the rotation: each score moves by up to 2 u sum |q||k| scale, which moves a
            # probability by twice that; then the probabilities' and the result's rounding
            u = 2.0 ** -8
            ds = (torch.einsum("ihgd,jhd->hgij", qq.abs().view(z - a, 2, 3, 64), kk.abs()) * scale * 2 * u).amax(-1)
            tol = u * want.abs() + size * (u + 2 * ds.permute(2, 0, 1).reshape(z - a, hq, 1) + 1e-4) * 1.02
            assert not bool(((o.double() - want).abs() > tol).any())

    eng.spawn(0)
    eng.append(0, tokens[:500])
    eng.map_blocks([0], B.MAP_LOOKUP)
    eng.map_blocks([0], B.MAP_ADMIT)
    chunk(0, 0, 333)
    chunk(0, 333, 500)                  # ends inside a block: 4 tokens in the tail block
    eng.prefill_done(0)
    victims, _ = eng.select_victims(B.TIER_HBM, 40)
    rc, done, _ = eng.offload(victims)
    assert rc == 0 and done == 31
    eng.spawn(1)                        # somebody else takes the low slots meanwhile
    eng.append(1, tokens[::-1][:100].copy())
    eng.map_blocks([1], B.MAP_LOOKUP)
    eng.map_blocks([1], B.MAP_ADMIT)
    eng.append(0, tokens[500:520])
    info = eng.map_blocks([0], B.MAP_LOOKUP)
    assert int(info["n_hit_host"][0]) == 31
    _, tier, slot = eng.get_block_map(0)
    rc, done = eng.reload(slot[tier == B.TIER_HOST])
    assert rc == 0 and done == 31
    eng.map_blocks([0], B.MAP_ADMIT)
    chunk(0, 496, 520)                  # the turn's tokens, and again those that had no full block
    for t in range(520, 523):           # decode: token by token into the tail block
        chunk(0, t, t + 1)
    eng.close()
