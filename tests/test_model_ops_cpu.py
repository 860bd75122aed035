"""What of append_kv and attend can be checked without a GPU: struct layouts, NULL arguments, the Rope description."""
import ctypes as C
import re
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIZES = {"uint32_t": 4, "uint64_t": 8, "float": 4, "pointer": 8}


def header_struct(name):
    """(field, size) in the header's order, nested batch included as one field."""
    text = open(os.path.join(ROOT, "include", "kvt.h")).read()
    body = text[text.index(f"typedef struct {name} {{"):text.index(f"}} {name};")]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S).split("{", 1)[1]
    out = []
    for decl in body.split(";"):
        m = re.match(r"\s*(?:const\s+)?(\w+)\s+(.*)", decl.strip(), flags=re.S)
        if not m:
            continue
        for x in m.group(2).split(","):
            x = x.strip()
            out.append((x.lstrip("*"), 8 if x.startswith("*") else SIZES.get(m.group(1), 0)))
    return out


@pytest.mark.parametrize("name,cls", [("kvt_batch", "Batch"), ("kvt_append_args", "AppendArgs"), ("kvt_attend_args", "AttendArgs")])
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
    a, t = B.AppendArgs(), B.AttendArgs()
    assert lib.kvt_append_kv(None, C.byref(a), None) == B.E_INVAL
    assert lib.kvt_attend(None, C.byref(t), None) == B.E_INVAL
    assert lib.kvt_attend_scratch_bytes(None, C.byref(t)) == 0
    assert lib.kvt_set_tail_pool(None, None, 0) == B.E_INVAL
    assert lib.kvt_kv_check(None, None) == B.E_INVAL


def test_rope_description():
    from paper_2609_39819_b200 import binding as B
    r = B.Rope(8, theta=100.0, sections=[1, 0, 3], device="cpu")
    assert r.n_axes == 3 and r.axis_of.tolist() == [0, 2, 2, 2]
    assert r.freqs.tolist() == pytest.approx([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], rel=1e-15)
    assert B.Rope(4, freqs=[1.0, 0.5], axis_of=[1, 0], device="cpu").n_axes == 2
    assert B.Rope(0, device="cpu").freqs.numel() == 0
    for bad in (dict(rot_dim=7), dict(rot_dim=8, sections=[1, 2]), dict(rot_dim=8, sections=[5, -1]),
                dict(rot_dim=8, freqs=[1.0]), dict(rot_dim=8, axis_of=[0, 1]), dict(rot_dim=4, axis_of=[0, 256]),
                dict(rot_dim=4, axis_of=[0, 1], sections=[1, 1])):
        with pytest.raises(ValueError):
            B.Rope(device="cpu", **bad)


def test_packed_arguments_are_the_structs():
    """The calls pack their arguments with struct; every field must land where the ctypes structs have it."""
    from paper_2609_39819_b200 import binding as B
    for cls, packer in ((B.AppendArgs, B._APPEND), (B.AttendArgs, B._ATTEND)):
        assert packer.size == C.sizeof(cls)
        names = [f[0] for f in B.Batch._fields_] + [f[0] for f in cls._fields_[1:]]
        x = cls.from_buffer_copy(packer.pack(*range(1, len(names) + 1)))
        got = [getattr(x.b, f[0]) for f in B.Batch._fields_] + [getattr(x, f[0]) for f in cls._fields_[1:]]
        assert got == list(range(1, len(names) + 1))


def test_native_marshalling_leaves_what_it_does_not_take_to_the_callers_checks():
    """Wrong numbers of arguments, types, devices and shapes: no call is made, nothing is raised, nothing read."""
    import torch
    from paper_2609_39819_b200 import binding
    native = binding.load_native()
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)      # noqa: E731
    append = [0, 0, 0, 0, 2, 64, 0, k, k, ints(0).view(1, 1), ints(0, 3), ints(3), 0, 1, None, None, False, None, None, None]
    attend = [0, 0, 0, 0, 0, 2, 64, 0, k, ints(0).view(1, 1), ints(0, 3), ints(3), None, True, None, None, None, None]
    for call, args in ((native.append, append), (native.attend, attend)):
        assert call(*args) is NotImplemented                  # tensors that are not on a CUDA device
        assert call() is NotImplemented and call(*args[:-1]) is NotImplemented
        for i in range(len(args)):
            for wrong in (None, -1, 1 << 70, "x", 1.5, k.float(), k[0], ints(1)):
                assert call(*args[:i], wrong, *args[i + 1:]) is NotImplemented


@pytest.fixture
def no_native_yet(monkeypatch):
    from paper_2609_39819_b200 import binding
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding, "_native_missing", None, raising=False)
    return binding


def test_without_the_native_marshalling_every_call_is_left_to_python(no_native_yet, monkeypatch):
    from paper_2609_39819_b200 import build
    tried = []

    def cannot(force=False):
        tried.append(1)
        raise OSError("no compiler")

    monkeypatch.setattr(build, "build_torch_lib", cannot)
    for _ in range(2):
        with pytest.warns(UserWarning, match="no compiler"):
            calls = no_native_yet._native_calls(no_native_yet.load_library())
        assert [f(1, 2, 3) for f in calls] == [NotImplemented, NotImplemented]
    assert len(tried) == 1          # an engine more does not try again for a minute
    with pytest.raises(RuntimeError, match="no compiler"):
        no_native_yet.load_native()


def test_the_native_marshalling_belongs_to_one_torch(no_native_yet, monkeypatch):
    import importlib.metadata
    import torch
    from paper_2609_39819_b200 import build
    assert torch.__version__ in build.TORCH_LIB
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "1.2.3")
    assert "1.2.3" in build._torch_lib() and not os.path.exists(build._torch_lib())


def test_the_attention_kernels_are_compiled_once_for_all_libraries(monkeypatch, tmp_path):
    from paper_2609_39819_b200 import build
    commands = []

    def compiler(cmd):
        commands.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build.subprocess, "check_call", compiler)
    monkeypatch.setattr(build, "ATTEND_OBJ", str(tmp_path / "attend.o"))
    for name, defines in (("a.so", None), ("b.so", ["-DKVT_DEBUG"]), ("c.so", ["-DKVT_TRACE"])):
        assert build.build_lib(lib=str(tmp_path / name), defines=defines) == str(tmp_path / name)
    of = lambda src: [c for c in commands if any(x.endswith(src) for x in c)]       # noqa: E731
    assert len(of("kvt_attend.cu")) == 1 and not any(x.startswith("-D") for x in of("kvt_attend.cu")[0])
    assert len(of("kvt_engine.cu")) == 3 and ["-DKVT_DEBUG" in c for c in of("kvt_engine.cu")] == [False, True, False]
    links = [c for c in commands if "-shared" in c]
    assert len(links) == 3 and all(str(tmp_path / "attend.o") in c for c in links)
    assert sorted(p.name for p in tmp_path.iterdir() if not p.name.endswith(".lock")) == ["a.so", "attend.o", "b.so", "c.so"]
