"""append_kv and attend where they are easily wrong: what lies just outside the rows' keys, the ends of the element types'
ranges, arguments that are nearly right, reports from several streams. Setup and its 64-bit reference are the other file's."""
import ctypes as C
import functools
import math
from types import SimpleNamespace

import pytest
from test_gpu_model_ops import B, BT, Setup  # noqa: F401  (B is a fixture)

pytestmark = pytest.mark.gpu


def every_kernel(s, **kw):
    """attend by everything the kernel is chosen by (as in check_attend): few rows, prompts, with and without parts."""
    wide = s.widened()
    for table, hint in ((s.table, max(s.new)), (wide, None), (s.table, 1), (wide, 1)):
        lse = s.torch.empty(s.rows, s.heads * s.group, device="cuda")
        yield (table is wide, hint), s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len, max_q_len=hint, lse=lse, **kw), lse
    s.eng.kv_check()


def cached(s, i, c):
    """(layer's K or V by slot, slots) of sequence i: blocks as [block, 16, heads, dim] by pool[slots]."""
    n = -(-s.kv[i] // BT)
    return s.pools[0][2 * s.layer + c], s.host_table[i, :n].long().cuda()


# ---- fp16: small probabilities that a long context adds up ------------------------------------------------------
def sink_case(s, gap, sinks, value, seed):
    """Scores in powers of two (scale ln 2): `sinks` hold 0 and a value of 0, all other keys -gap with some spread and values
    around `value`. Returns out and lse in 64 bits and by how much they may be off."""
    torch = s.torch
    g = torch.Generator("cuda").manual_seed(seed)
    n = s.kv[0]
    s.q.zero_()
    s.q[..., 0] = 1.0
    score = -gap + torch.randint(-32, 33, (n,), generator=g, device="cuda") / 64.0       # exact in fp16 for gaps below 32
    score[[x for x in sinks if x < n]] = 0.0
    v = (torch.rand(n, s.heads, s.dim, generator=g, device="cuda") + 0.5) * value
    v[[x for x in sinks if x < n]] = 0.0
    for c, x in ((0, torch.zeros_like(v)), (1, v)):
        if c == 0:
            x[..., 0] = score[:, None]
        full = torch.full((-(-n // BT) * BT, s.heads, s.dim), math.nan, device="cuda")
        full[:n] = x
        pool, slots = cached(s, 0, c)
        pool[slots] = full.view(-1, BT, s.heads, s.dim).to(s.dt)
    k, v = s.gather(0)
    x = k[:, :, 0].T[:, None, :] * 1.0                                                    # [heads, 1, keys]
    own = torch.arange(n - s.new[0], n, device="cuda")
    x = torch.where(torch.arange(n, device="cuda")[None] <= own[:, None], x, -math.inf)  # [heads, rows, keys]
    p = torch.exp2(x)
    total = p.sum(-1)
    out = torch.einsum("hij,jhd->ihd", p, v) / total.T[..., None]
    # The powers' own rounding (once to fp16, where there are many rows) and the result's: u each. A power is relative to a number
    # that leaves the largest one of 128 keys at 2^-4 or more, where fp16 has a fixed step of 2^-24: 128 * 2^-25 * 2^4 of
    # the step's sum, three times that as values differ by 3. Keys beside a sink are relative to the sink's 2^8. Sums of N keys:
    # the matrix units add 16 products at a time and may cut off what is below 2^-23 of the sum (N / 16 times), denominators
    # are added up one by one from eight keys of four warps. Scores: a product by ln 2 * log2 e, 32 units at most.
    rel = 2 * s.u + 3 * 2.0 ** -14 + (n / 16 + 64) * 2.0 ** -23 + n * 2.0 ** -27 + 64 * 2.0 ** -24
    tol = rel * out + len(sinks) * 128 * 1.5 * value * 2.0 ** -33 + 2.0 ** -25
    tol_l = torch.full_like(total.T, (n * 2.0 ** -27 + 2.0 ** -16))
    hq = s.heads * s.group
    rep = lambda y: y.repeat_interleave(s.group, 1)          # noqa: E731
    assert out.shape[1] * s.group == hq
    return rep(out), rep(torch.log(total).T), rep(tol), rep(tol_l)


@pytest.mark.parametrize("dim", [64, 128, 72])
@pytest.mark.parametrize("new,past,gap,value", [(1, 100_000, 22, 1.0), (1, 100_000, 25, 1.0), (60, 100_000, 26, 1.0), (1, 4000, 25, 1.0),
                                                (60, 4000, 25, 1.0), (1, 130_000, 31, 1024.0), (60, 30_000, 28, 32000.0),
                                                (1, 60_000, 14, 1.0), (60, 60_000, 18, 1.0)])
@pytest.mark.parametrize("where", ["first", "last", "both and between"])
def test_fp16_sums_what_is_far_below_the_largest_score(B, dim, new, past, gap, value, where):  # noqa: F811
    """A key that takes nearly all of the weight and has nothing to say (an attention sink): the result is what the others add up to."""
    import torch
    s = Setup(B, [new], [past], heads=1, group=4, dim=dim, dtype="fp16", layers=1, layer=0, seed=past + gap)
    n = s.kv[0]
    sinks = {"first": [0], "last": [past - 1], "both and between": [0, past // 3, past // 3 + 1, past // 2, past - 1]}[where]
    want, wl, tol, tl = sink_case(s, gap, sinks, value, past + gap)
    for which, got, lse in every_kernel(s, scale=math.log(2.0)):
        bad = (got.double() - want).abs() > tol
        assert not bool(bad.any()), (which, n, float(((got.double() - want).abs() / want).max()))
        assert not bool(((lse.double() - wl).abs() > tl).any()), (which, float((lse.double() - wl).abs().max()))


def test_fp16_scores_that_go_up_and_down_by_much(B):  # noqa: F811
    """Every block of keys on another level, up to 200 binades apart, rising, falling and in turn."""
    import torch
    for dim in (64, 128, 72):
        for new in (1, 60):
            for kind in ("down", "up", "turns"):
                s = Setup(B, [new], [9000], heads=1, group=4, dim=dim, dtype="fp16", layers=1, layer=0, seed=dim + new)
                s.put()
                n = s.kv[0]
                b = torch.arange(n, device="cuda") // BT
                level = {"down": -200.0 * b / b.max(), "up": 200.0 * b / b.max(), "turns": -((b * 37) % 60).float()}[kind]
                pool, slots = cached(s, 0, 0)
                k = torch.zeros(len(slots) * BT, 1, dim, device="cuda")
                k[:n, 0, 0] = (level * 8).round() / 8
                pool[slots] = k.view(-1, BT, 1, dim).to(s.dt)
                s.q.zero_()
                s.q[..., 0] = 1.0
                want, wl, tol, tl = s.reference(scale=math.log(2.0))
                a = []
                for which, got, lse in every_kernel(s, scale=math.log(2.0)):
                    bad = (got.double() - want).abs() > tol
                    assert not bool(bad.any()), (dim, new, kind, which)
                    assert not bool(((lse.double() - wl).abs() > tl + 220 * 2.0 ** -23).any()), (dim, new, kind, which)   # log2 of a sum of 2^200
                    a.append(got)


# ---- keys that nobody sees ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 72, 20])
@pytest.mark.parametrize("new,past,window", [(1, 300, 100), (1, 1500, 1003), (40, 300, 9), (200, 700, 333), (200, 2500, 1000), (1, 30, 2)])
def test_values_in_front_of_a_window_have_no_effect(B, new, past, window, dim, dtype):  # noqa: F811
    """The block of the first key that is seen begins with tokens that no row sees: NaN or Inf there must not get anywhere."""
    import torch
    s = Setup(B, [new, 3], [past, past // 2], heads=2, group=2, dim=dim, dtype=dtype, seed=past + window)
    s.put()
    want = [(got.clone(), lse.clone()) for _, got, lse in every_kernel(s, window=window)]
    spoiled = 0
    for bad in (math.nan, math.inf, -math.inf):
        for i, (n, kv) in enumerate(zip(s.new, s.kv)):
            first = max(0, kv - n + 1 - window)
            at = first // BT * BT
            for t in range(at, first):
                for c in (0, 1):
                    s._chunk(int(s.host_table[i, t // BT]), c)[t % BT] = bad
                spoiled += 1
        for (which, got, lse), (w, wl) in zip(every_kernel(s, window=window), want):
            assert torch.equal(got, w) and torch.equal(lse, wl), (which, bad)
    assert spoiled


# ---- reports ---------------------------------------------------------------------------------------------------------
def test_no_report_is_lost_between_two_streams(B):  # noqa: F811
    """Bad slots met on one stream while kv_check runs on another, over and over: each is reported once."""
    import time
    import torch
    s = Setup(B, [1], [40], heads=1, group=1, dim=64, seed=3)
    bad = torch.full_like(s.table, 0x7FFFFFF0)
    other = torch.cuda.Stream()
    s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len)
    s.eng.kv_check()
    torch.cuda.synchronize()
    lost = 0
    for i in range(400):
        with torch.cuda.stream(other):
            torch.cuda._sleep(20000 + 997 * (i % 50))
            s.eng.append_kv(s.layer, s.k, s.v, bad, s.q_start, s.kv_len)
            done = torch.cuda.Event()
            done.record()
        reports, late = 0, 0
        while late < 3:                     # three checks begun after the bad call was through
            late += done.query()
            try:
                s.eng.kv_check()
            except B.KvtError as exc:
                assert exc.code == B.E_RANGE
                reports += 1
        assert reports <= 1
        lost += reports == 0
    assert lost == 0


# ---- marshalling -----------------------------------------------------------------------------------------------------
def test_an_engine_without_the_native_marshalling(B, monkeypatch):  # noqa: F811
    """The native module saves host time and nothing else: without it engines are made and give the same results."""
    import torch

    def missing():
        raise RuntimeError("no module")

    with_it = Setup(B, [5, 40], [30, 200], heads=2, group=2, dim=64, seed=8)
    monkeypatch.setattr(B, "load_native", missing)
    with pytest.warns(UserWarning, match="no module"):
        meta = B.Engine(n_layers=2, n_kv_heads=2, head_dim=64, n_hbm_blocks=8, n_host_blocks=0, metadata_only=True, max_tokens=256)
    meta.spawn(0)
    with pytest.warns(UserWarning, match="no module"):
        without = Setup(B, [5, 40], [30, 200], heads=2, group=2, dim=64, seed=8)
    got = []
    for s in (with_it, without):
        q = s.eng.append_kv(s.layer, s.k, s.v, s.table, s.q_start, s.kv_len, rope=B.Rope(64), q=s.q)
        got.append((q, s.eng.attend(s.layer, q, s.table, s.q_start, s.kv_len), *s.bits()))
        s.eng.kv_check()
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_scale_of_nothing(B):  # noqa: F811
    """scale=0.0 is a scale, not the default: all keys weigh the same. So does one that is 0 in 32 bits."""
    import torch
    for dim in (64, 72):
        s = Setup(B, [1, 30], [50, 300], heads=2, group=2, dim=dim, seed=5)
        s.put()
        for scale in (0.0, 0, -0.0, 1e-60):
            want, wl, tol, tl = s.reference(scale=0.0)
            for _, got, lse in every_kernel(s, scale=scale):
                assert not bool(((got.double() - want).abs() > tol).any())
                assert not bool(((lse.double() - wl).abs() > tl).any())


def test_inputs_that_require_gradients_are_refused(B):  # noqa: F811
    """There is no backward pass: results that silently carry no gradient are not what such a caller wants."""
    import torch
    s = Setup(B, [4], [20], heads=1, group=2, dim=64, seed=6)
    good = (s.table, s.q_start, s.kv_len)
    leaf = lambda x: x.detach().clone().requires_grad_()          # noqa: E731
    for native in (True, False):
        if not native:
            s.eng._append_native = s.eng._attend_native = lambda *a: NotImplemented
        for f in (lambda: s.eng.attend(s.layer, leaf(s.q), *good), lambda: s.eng.append_kv(s.layer, leaf(s.k), s.v, *good),
                  lambda: s.eng.append_kv(s.layer, s.k, leaf(s.v), *good),
                  lambda: s.eng.append_kv(s.layer, s.k, s.v, *good, rope=B.Rope(64), q=leaf(s.q)),
                  lambda: s.eng.attend(s.layer, s.q, *good, out=leaf(s.q))):
            with pytest.raises(ValueError, match="gradient"):
                f()
        with torch.no_grad():
            s.eng.append_kv(s.layer, leaf(s.k), leaf(s.v), *good)
            a = s.eng.attend(s.layer, leaf(s.q), *good)
        assert torch.equal(a, s.eng.attend(s.layer, s.q, *good)) and not a.requires_grad
    s.eng.kv_check()


def test_tail_pool_of_another_device_is_refused(B):  # noqa: F811
    import torch
    s = Setup(B, [4], [20], heads=1, group=2, dim=64, tail=True, seed=6)
    p = s.eng.tail_pool
    elsewhere = SimpleNamespace(device=torch.device("cuda", s.eng._dev_index + 1), dtype=p.dtype, is_contiguous=lambda: True,
                                data_ptr=p.data_ptr, numel=p.numel, get_device=lambda: s.eng._dev_index + 1)
    with pytest.raises(ValueError, match="device"):
        s.eng.set_tail_pool(elsewhere)
    with pytest.raises(ValueError, match="device"):
        s.eng.set_tail_pool(torch.zeros(p.numel(), dtype=torch.uint8))
    assert s.eng.tail_pool is p


def test_positions_and_tables_that_are_broadcast(B):  # noqa: F811
    """One row of positions for all axes (text among images), one table row for all sequences: read only, so nothing to refuse."""
    import torch
    s = Setup(B, [7, 20], [50, 3], heads=2, group=2, dim=64, seed=7)
    rope = B.Rope(64, sections=[12, 10, 10])
    pos = torch.arange(s.t, dtype=torch.int32, device="cuda") * 11
    args = (s.table, s.q_start, s.kv_len)
    for native in (True, False):
        if not native:
            s.eng._append_native = s.eng._attend_native = lambda *a: NotImplemented
        want = s.eng.append_kv(s.layer, s.k, s.v, *args, rope=rope, positions=pos.repeat(3, 1), q=s.q)
        pool = s.bits()
        got = s.eng.append_kv(s.layer, s.k, s.v, *args, rope=rope, positions=pos[None].expand(3, -1), q=s.q)
        assert torch.equal(want, got) and all(torch.equal(a, b) for a, b in zip(pool, s.bits()))
        shared = s.table[:1].expand(2, -1)
        short = torch.full_like(s.kv_len, min(s.kv))
        assert torch.equal(s.eng.attend(s.layer, s.q, shared, s.q_start, short),
                           s.eng.attend(s.layer, s.q, shared.contiguous(), s.q_start, short))
    s.eng.kv_check()


def test_scratch_that_is_too_small_or_misaligned(B):  # noqa: F811
    s = Setup(B, [100, 5], [3000, 40], heads=2, group=2, dim=128, seed=9)
    out = s.torch.empty_like(s.q)
    table = s.widened()                             # rows that could hold 320 K tokens: sequences may have to be cut
    a = B.AttendArgs(B.Batch(2, s.t, table.shape[1], 0, table.stride(0), s.q_start.data_ptr(), s.kv_len.data_ptr(), table.data_ptr()),
                     s.layer, 0, 4, 0, 0, 0.0, s.q.data_ptr(), out.data_ptr(), None, *s.q.stride()[:2], *out.stride()[:2])
    lib, h = s.eng.L, s.eng.h
    need = lib.kvt_attend_scratch_bytes(h, C.byref(a))
    assert need > 0
    scratch = s.torch.empty(need + 16, dtype=s.torch.uint8, device="cuda")
    for ptr, size, code in ((scratch.data_ptr(), need - 1, B.E_BUFSZ), (None, need, B.E_BUFSZ), (scratch.data_ptr(), 0, B.E_BUFSZ),
                            (scratch.data_ptr() + 8, need, B.E_INVAL)):
        a.scratch, a.scratch_bytes = ptr, size
        assert lib.kvt_attend(h, C.byref(a), None) == code
    a.scratch, a.scratch_bytes = scratch.data_ptr(), need
    s.put()
    s.torch.cuda.synchronize()                      # this call runs on the default stream
    assert lib.kvt_attend(h, C.byref(a), None) == 0
    s.torch.cuda.synchronize()
    s.eng.kv_check()
    assert s.torch.equal(out, s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len))


def test_one_wrong_argument_at_a_time(B):  # noqa: F811
    """From calls that are taken, one argument spoiled: neither marshalling makes the call. (The library's entry points are stood in
    for, so that nothing runs whatever gets through.)"""
    import torch
    s = Setup(B, [3, 5], [30, 200], heads=2, group=2, dim=64, seed=8)
    t, cuda = s.t, dict(device="cuda")
    made = []
    entry = C.CFUNCTYPE(C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p)(lambda e, a, st: made.append(1) or 0)
    bytes_ = C.CFUNCTYPE(C.c_uint64, C.c_void_p, C.c_void_p)(lambda e, a: 0)
    at = lambda f: C.cast(f, C.c_void_p).value               # noqa: E731
    s.eng._append_native = functools.partial(B.load_native().append, at(entry))
    s.eng._attend_native = functools.partial(B.load_native().attend, at(entry), at(bytes_))
    real = s.eng.L
    rope = B.Rope(64, sections=[8, 24])
    pos = torch.zeros(2, t, dtype=torch.int32, **cuda)
    lse = torch.zeros(t, 4, **cuda)

    def other(x):
        return [x.cpu(), x.float() if x.dtype != torch.float32 else x.half(), x[..., None], x[0], x[:, :1].repeat(1, 7)[:, :x.shape[1] - 1]
                if x.dim() == 2 else x[:-1]]

    append = dict(layer=s.layer, k=s.k, v=s.v, block_table=s.table, q_start=s.q_start, kv_len=s.kv_len, rope=rope, positions=pos, q=s.q,
                  q_out=torch.zeros_like(s.q))
    attend = dict(layer=s.layer, q=s.q, block_table=s.table, q_start=s.q_start, kv_len=s.kv_len, max_q_len=5, causal=True, window=7,
                  scale=0.5, out=torch.zeros_like(s.q), lse=lse)
    spoilt = {
        "layer": [-1, None, "x", 1 << 70], "k": other(s.k) + [None, s.k[..., ::2], s.k.half()], "v": other(s.v) + [None, s.v.half()],
        "block_table": [s.table.cpu(), s.table.long(), s.table[0], s.table[:1], s.table.T.contiguous().T, None],
        "q_start": [s.q_start.cpu(), s.q_start.long(), s.q_start[:-1], s.q_start[None], s.q_start.repeat_interleave(2)[::2], None],
        "kv_len": [s.kv_len.cpu(), s.kv_len.long(), s.kv_len[:-1], s.kv_len[None], s.kv_len.repeat_interleave(2)[::2], None],
        "positions": [None, pos.cpu(), pos.long(), pos[:1], pos[0], pos[:, :-1], pos.T.contiguous().T],
        "rope": [None, B.Rope(64, sections=[8, 20, 4])],
        "q": [s.q.cpu(), s.q.float(), s.q.half(), s.q[0], s.q[:-1], s.q[..., :32]],
        "q_out": other(s.q) + [s.q[:, :1].expand(-1, 4, -1), s.q[:1].expand(t, -1, -1)],
        "out": other(s.q) + [s.q[:, :1].expand(-1, 4, -1), s.q[:1].expand(t, -1, -1)],
        "lse": other(lse) + [torch.zeros(4, t, **cuda).T, lse.half()],
        "max_q_len": [-1, "x"], "window": [-1, "x"], "scale": ["x"],
    }
    for call, args in ((s.eng.append_kv, append), (s.eng.attend, attend)):
        which = "_append_native" if call == s.eng.append_kv else "_attend_native"
        native = getattr(s.eng, which)
        for python in (False, True):
            s.eng.L = SimpleNamespace(kvt_append_kv=lambda e, a, st: made.append(1) or 0, kvt_attend=lambda e, a, st: made.append(1) or 0,
                                      kvt_attend_scratch_bytes=lambda e, a: 0)
            setattr(s.eng, which, (lambda *a: NotImplemented) if python else native)
            try:
                call(**args)
                assert made == [1]
                made.clear()
                for name in args:
                    for i, wrong in enumerate(spoilt.get(name, [])):
                        with pytest.raises(Exception):
                            call(**{**args, name: wrong})
                        assert not made, (name, i, python)
                    made.clear()
            finally:
                s.eng.L = real
                setattr(s.eng, which, native)


# ---- very long work ------------------------------------------------------------------------------------------------------
def test_warps_wait_as_long_as_a_job_takes(B):  # noqa: F811
    """A job of more than a second in front of a short one: the warps that wait for the short one must not give up. 130 M
    cached tokens of 148 heads, whose table row names the same 60 blocks over and over."""
    import torch
    heads, group, dim, n_slots, long_kv = 148, 4, 64, 64, 130_000_000
    eng = B.Engine(n_layers=1, n_kv_heads=heads, head_dim=dim, n_hbm_blocks=n_slots, n_host_blocks=0, max_contexts=1, max_messages=16,
                   max_tokens=64)
    g = torch.Generator("cuda").manual_seed(1)
    eng.hbm_pool.view(torch.bfloat16).normal_(generator=g)
    new, kv = [32, 64], [long_kv, 500]              # one tile of rows, then two
    q = torch.randn(sum(new), heads * group, dim, generator=g, device="cuda").bfloat16()
    table = (torch.arange(-(-long_kv // BT), device="cuda") % 60).int()[None].expand(2, -1)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")          # noqa: E731
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    out = eng.attend(0, q, table, ints(0, 32, 96), ints(*kv), max_q_len=64)
    end.record()
    eng.kv_check()
    assert begin.elapsed_time(end) > 1000, "not as long as it has to be for this test"
    assert bool(torch.isfinite(out).all())
    pool = eng.hbm_pool.view(torch.bfloat16).view(2, n_slots, BT, heads, dim).double()
    k, v = (pool[c, :60].reshape(-1, heads, dim)[:500].repeat_interleave(group, 1) for c in (0, 1))
    x = torch.einsum("ihd,jhd->hij", q[32:].double(), k) * dim ** -0.5
    x = x.masked_fill(torch.arange(500, device="cuda")[None] > torch.arange(436, 500, device="cuda")[:, None], -math.inf)
    p = torch.softmax(x, -1)
    want, size = torch.einsum("hij,jhd->ihd", p, v), torch.einsum("hij,jhd->ihd", p, v.abs())
    # the probabilities' and the result's rounding, and 32-bit sums of 500 terms and scores of 64
    assert not bool(((out[32:].double() - want).abs() > 2.0 ** -8 * want.abs() + size * (2.0 ** -8 + 2.0 ** -12)).any())
    eng.close()


# ---- rounding ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 72])
@pytest.mark.parametrize("past", [5, 300, 3000])
def test_few_rows_are_as_exact_as_with_32_bit_probabilities(B, past, dim, dtype):  # noqa: F811
    """Only the result is rounded to the element type, not the probabilities."""
    import torch
    s = Setup(B, [2], [past], heads=2, group=3, dim=dim, dtype=dtype, seed=past + dim)
    s.put()
    n = s.kv[0]
    k, v = (x.repeat_interleave(3, 1) for x in s.gather(0))
    q = s.q.double()
    x = torch.einsum("ihd,jhd->ihj", q, k) * dim ** -0.5
    hidden = torch.arange(n, device="cuda")[None, None] > torch.arange(n - 2, n, device="cuda")[:, None, None]
    p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
    want, size = torch.einsum("ihj,jhd->ihd", p, v), torch.einsum("ihj,jhd->ihd", p, v.abs())
    # scores: dim products summed in 32 bits and the scaling; sums over the keys in 32 bits; a probability is the sum of two numbers,
    # the second rounded: u * u, or for fp16 (16 keys' fixed step, 2^-25 each, relative to 2^-4 at least) 2^-17 of the largest
    big = (torch.einsum("ihd,jhd->ihj", q.abs(), k.abs()) * dim ** -0.5).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
    rel = 2 * (dim + 4) * 2.0 ** -24 * big + 2 * (n + 64) * 2.0 ** -24 + max(s.u * s.u, 2.0 ** -17)
    tol = s.u * want.abs() + size * rel * (1 + s.u) + (2.0 ** -25 if dtype == "fp16" else 0.0)
    assert dtype == "fp16" or bool((rel < s.u / 3).all())      # so that probabilities rounded once would show
    for table in (s.table, s.widened()):
        got = s.eng.attend(s.layer, s.q, table, s.q_start, s.kv_len, max_q_len=2)
        bad = (got.double() - want).abs() > tol
        assert not bool(bad.any()), int(bad.sum())
    s.eng.kv_check()


@pytest.mark.parametrize("dim", [64, 128, 72])
@pytest.mark.parametrize("new", [1, 40, 200])
def test_fp16_nan_and_infinite_scores_stay_with_the_rows_that_see_them(B, new, dim):  # noqa: F811
    """NaN and +Inf spoil the rows that see the key, -Inf takes its weight away; what the powers are relative to survives all of them."""
    import torch
    for back in (0, 7, 120, 250):                   # how far before the end the key lies
        s = Setup(B, [new, 5], [300, 40], heads=2, group=2, dim=dim, dtype="fp16", seed=9)
        s.q[:, :, 0] = s.q[:, :, 0].abs() + 0.5
        s.put()
        at = s.kv[0] - 1 - back
        place = s._chunk(int(s.host_table[0, at // BT]), 0)[at % BT, 1]
        spoilt = torch.zeros(s.t, 4, dtype=torch.bool, device="cuda")
        spoilt[:new, 2:] = (torch.arange(new, device="cuda") + 300 >= at)[:, None]
        for bad in (math.nan, math.inf, -math.inf):
            place[0] = bad
            for _, got, lse in every_kernel(s):
                if bad == -math.inf:
                    assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(lse).all()), (back, bad)
                else:
                    assert torch.equal(torch.isnan(got).all(-1), spoilt) and torch.equal(torch.isfinite(got).all(-1), ~spoilt), (back, bad)
                    assert torch.equal(torch.isfinite(lse), ~spoilt), (back, bad)


def test_lse_that_requires_a_gradient_is_refused(B):  # noqa: F811
    import torch
    s = Setup(B, [4], [20], heads=1, group=2, dim=64, seed=6)
    for native in (True, False):
        if not native:
            s.eng._attend_native = lambda *a: NotImplemented
        with pytest.raises(ValueError, match="gradient"):
            s.eng.attend(s.layer, s.q, s.table, s.q_start, s.kv_len, lse=torch.zeros(4, 2, device="cuda", requires_grad=True))
