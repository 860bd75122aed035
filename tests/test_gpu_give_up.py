"""What the model-side kernels do where a wait inside them runs out: they end, say so, and read and write nothing outside their arrays."""
import ctypes as C
import math

import pytest

from test_gpu_model_ops import B, Setup  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64)])
def test_attend_that_gives_up_a_wait(B, dtype, dim):  # noqa: F811
    """70 sequences, the first of them cut into pieces, 8 KV heads: the planning warp gives up before it has planned the last sequences, whose
    plans then hold what the scratch held before, here all ones. Their parts are not looked for."""
    import torch
    n = 70
    s = Setup(B, [300] * n, [100000] + [50 * i % 900 for i in range(1, n)], 8, 4, dim, dtype, layers=1, layer=0)
    s.put()
    guard = 7.25
    out = torch.full((s.t + 1, 32, dim), guard, dtype=s.dt, device="cuda")
    b = B.Batch(*s.eng._kv_batch("", s.t, s.table, s.q_start, s.kv_len, 300))
    strides = (*s.q.stride()[:2], *out.stride()[:2])
    a = B.AttendArgs(b, 0, 0 if dtype == "bf16" else 1, 32, 0, 0, 0.0, s.q.data_ptr(), out.data_ptr(), 0, *strides, 0, 0)
    size = s.eng.L.kvt_attend_scratch_bytes(s.eng.h, C.byref(a))
    assert size
    scratch = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    a.scratch, a.scratch_bytes = scratch.data_ptr(), size
    before = s.eng.hbm_pool.clone()
    s.eng.set_wait_limit(0)
    assert s.eng.L.kvt_attend(s.eng.h, C.byref(a), s.eng._kv_stream()) == 0
    with pytest.raises(B.KvtError, match="wait"):
        s.eng.kv_check()
    assert torch.equal(before, s.eng.hbm_pool) and bool((out[s.t:] == guard).all()) and bool((scratch[size:] == 255).all())
    plans = scratch[:16 * (n + 1)].view(torch.int32).view(n + 1, 4).tolist()         # a header, then {first part, pieces, tiles, -} of each
    assert plans[0][0] == 1 and plans[1][1] > 1 and plans[n] == [-1] * 4             # the first is in pieces, the last has no plan
    s.eng.set_wait_limit(1 << 18)
    want = s.eng.attend(0, s.q, s.table, s.q_start, s.kv_len, max_q_len=300)
    assert s.eng.L.kvt_attend(s.eng.h, C.byref(a), s.eng._kv_stream()) == 0
    s.eng.kv_check()
    assert torch.equal(out[:s.t], want) and math.isfinite(float(out[:s.t].float().sum()))
