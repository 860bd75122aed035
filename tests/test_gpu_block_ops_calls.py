"""How the calls that choose blocks are made: by the native marshalling, and by one engine on two streams at once."""
import pytest

from test_gpu_block_ops import make, random_bounds
from test_gpu_model_ops import B, Setup  # noqa: F401

pytestmark = pytest.mark.gpu
NAMES = ("bound", "select", "attend_blocks", "weigh", "evict")


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("fp16", 40)])
def test_native_marshalling_runs_and_agrees_with_pythons(B, monkeypatch, dtype, dim):  # noqa: F811
    """Every call is taken by the native marshalling, and comes to the same as the one in Python, bounds included."""
    import torch
    s = make(B, ([40, 1], [900, 2000]), dtype, 0, 2, 4, dim, tail=True, strided=True)
    batch = (s.table, s.q_start, s.kv_len)
    lse = torch.full((s.t, 8), 6.0, device="cuda")
    old = torch.rand(s.table.shape, generator=torch.Generator("cuda").manual_seed(2), device="cuda")
    taken = {}

    def run():
        k = s.eng.key_bounds(s.dt)
        s.eng.bound_keys(s.layer, k, *batch, n_tokens=s.t)
        results = [k.codes.clone(), k.exps.clone()]
        assert int(k.codes.count_nonzero()) and int(k.exps.count_nonzero())
        k.codes.random_(-127, 128, generator=torch.Generator("cuda").manual_seed(1))
        k.exps.fill_(120)
        out_lse = torch.empty_like(lse)
        blocks = s.eng.select_blocks(s.layer, s.q, k, *batch, 12, first=2, last=3, max_q_len=40)
        results += [blocks, s.eng.attend_blocks(s.layer, s.q, blocks, *batch, scale=0.25, lse=out_lse), out_lse]
        for full in (False, True):
            results.append(s.eng.weigh_blocks(s.layer, s.q, lse, *batch, max_q_len=40, causal=not full, window=None if full else 500, scale=0.25,
                                              weights=old, keep=0.5))
        return results + list(s.eng.evict_blocks(old, s.table, s.kv_len, 20, first=3, last=4))

    def watch(name, call):
        def run_it(*args):
            done = call(*args)
            taken[name] = taken.get(name, True) and done is not NotImplemented
            return done
        return run_it

    for name in NAMES:
        monkeypatch.setattr(s.eng, f"_{name}_native", watch(name, getattr(s.eng, f"_{name}_native")))
    want = run()
    assert taken == {name: True for name in NAMES}
    for name in NAMES:
        monkeypatch.setattr(s.eng, f"_{name}_native", lambda *args: NotImplemented)
    for x, y in zip(want, run(), strict=True):
        assert torch.equal(x, y)
    s.eng.kv_check()


def test_one_engine_on_two_streams(B):  # noqa: F811
    """Sequences of one engine stepped by two streams at once, each with its own results: the same as one after the other."""
    import torch
    s = make(B, ([1, 60, 1, 200], [5000, 3000, 300, 100]), "bf16", 0, 2, 4, 128, layers=1, layer=0)
    eng = s.eng
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    chosen = random_bounds(s, torch.Generator("cuda").manual_seed(3))
    fresh = eng.key_bounds(s.dt)
    halves = []
    for a in (0, 2):                         # two sequences each
        t0, n = sum(s.new[:a]), s.new[a:a + 2]
        halves.append((s.q[t0:t0 + sum(n)], (s.table[a:a + 2], ints(0, n[0], sum(n)), ints(*s.kv[a:a + 2]))))

    def step(q, batch):
        eng.bound_keys(0, fresh, *batch, n_tokens=len(q))
        blocks = eng.select_blocks(0, q, chosen, *batch, 9)
        sparse = eng.attend_blocks(0, q, blocks, *batch)
        lse = torch.empty(len(q), 8, device="cuda")
        dense = eng.attend(0, q, *batch, lse=lse)
        weights = eng.weigh_blocks(0, q, lse, *batch)
        return (blocks, sparse, dense, lse, weights, *eng.evict_blocks(weights, *batch[::2], 9))

    want = [step(*h) for h in halves]
    bounds = (fresh.codes.clone(), fresh.exps.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        fresh.codes.zero_()
        fresh.exps.zero_()
        torch.cuda.synchronize()
        got = [None, None]
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                got[i] = step(*halves[i])
        torch.cuda.synchronize()
        for x, y in zip(want, got):
            assert all(torch.equal(a, b) for a, b in zip(x, y, strict=True))
        assert torch.equal(fresh.codes, bounds[0]) and torch.equal(fresh.exps, bounds[1])
    eng.kv_check()
