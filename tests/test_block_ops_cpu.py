"""What of the calls that choose blocks can be checked without a GPU: struct layouts, NULL arguments, the native marshalling's refusals."""
import ctypes as C

import pytest

from test_model_ops_cpu import header_struct


@pytest.mark.parametrize("name,cls", [("kvt_key_bounds", "KeyBoundsArgs"), ("kvt_bound_args", "BoundArgs"), ("kvt_select_args", "SelectArgs"),
                                      ("kvt_attend_blocks_args", "AttendBlocksArgs"), ("kvt_weigh_args", "WeighArgs"), ("kvt_evict_args", "EvictArgs")])
def test_structs_follow_the_header(name, cls):
    from paper_2609_39819_b200 import binding
    want = header_struct(name)
    got = getattr(binding, cls)._fields_
    assert [f for f, _ in want] == [f[0] for f in got]
    for (_, size), (_, ctype) in zip(want, got):
        assert size in (0, C.sizeof(ctype))


def test_null_arguments():
    from paper_2609_39819_b200 import binding as B
    lib = B.load_library()
    for call, args in (("bound_keys", B.BoundArgs()), ("select_blocks", B.SelectArgs()), ("attend_blocks", B.AttendBlocksArgs()),
                       ("weigh_blocks", B.WeighArgs()), ("evict_blocks", B.EvictArgs())):
        assert getattr(lib, f"kvt_{call}")(None, C.byref(args), None) == B.E_INVAL
    assert lib.kvt_select_scratch_bytes(None, C.byref(B.SelectArgs())) == 0
    assert lib.kvt_weigh_scratch_bytes(None, C.byref(B.WeighArgs())) == 0


def test_native_marshalling_leaves_what_it_does_not_take_to_the_callers_checks():
    """Wrong numbers of arguments, types, devices and shapes: no call is made, nothing is raised, nothing read."""
    import torch
    from paper_2609_39819_b200 import binding
    native = binding.load_native()
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    codes, exps = torch.zeros(1, 5, 2, 2, 64, dtype=torch.int8), torch.zeros(1, 5, 2, dtype=torch.uint8)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)      # noqa: E731
    table, start, length = ints(0).view(1, 1), ints(0, 3), ints(3)
    lists, floats = torch.zeros(3, 2, 4, dtype=torch.int32), torch.zeros(3, 4)
    calls = {
        native.bound: [0, 0, 0, 0, 2, 64, 1, 0, 0, codes, exps, table, start, length, 3],
        native.select: [0, 0, 0, 0, 0, 2, 64, 1, 0, 0, q, codes, exps, table, start, length, 4, 1, 2, None, None],
        native.attend_blocks: [0, 0, 0, 0, 2, 64, 0, q, lists, table, start, length, None, None, None],
        native.weigh: [0, 0, 0, 0, 0, 2, 64, 0, q, floats, table, start, length, None, True, None, None, None, 1.0, None],
        native.evict: [0, 0, 0, 0, 2, 64, floats[:1, :1], table, length, 4, 1, 2],
    }
    for call, args in calls.items():
        assert call(*args) is NotImplemented                  # tensors that are not on a CUDA device
        assert call() is NotImplemented and call(*args[:-1]) is NotImplemented
        for i in range(len(args)):
            for wrong in (None, -1, 1 << 70, "x", 1.5, q.float(), q[0], ints(1)):
                assert call(*args[:i], wrong, *args[i + 1:]) is NotImplemented


def test_without_the_native_marshalling_every_call_is_left_to_python(monkeypatch):
    from paper_2609_39819_b200 import binding

    def cannot():
        raise RuntimeError("none")

    monkeypatch.setattr(binding, "load_native", cannot)
    assert [f(1, 2, 3) for f in binding._native_block_calls(binding.load_library())] == [NotImplemented] * 5
