"""Thin ctypes binding of libkvt.so: argument marshalling only (that of the model-side calls natively where _kvt_torch*.so can be had). Every stage of the path (hashing,
table lookup, classification, victim selection, block movement) runs in the library's CUDA kernels.
PyTorch is used for device / pinned memory and streams, nothing else. There is no CPU fallback:
loading fails loudly when the library or a CUDA device is missing."""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvt.so")
# KVT_LIB=<path>: load another build of the same sources instead (the checked build libkvt_debug.so, a traced build)
ALT_LIB = os.environ.get("KVT_LIB")

OK, E_INVAL, E_NOCTX, E_RANGE, E_STATE, E_NOSPACE, E_BUFSZ, E_DEVICE, E_CUDA = 0, -1, -2, -3, -4, -5, -6, -7, -8
TIER_HBM, TIER_HOST, TIER_REMOTE, TIER_NONE = 0, 1, 2, 0xFF
LAYOUT_LAYER_MAJOR, LAYOUT_BLOCK_MAJOR = 0, 1
ORDER_MRU, ORDER_LRU = 0, 1
POLICY_NO_LIFECYCLE, POLICY_INCLUSIVE, POLICY_ORPHANS_DEAD = 1, 2, 4
(OP_SPAWN, OP_FORK, OP_APPEND, OP_REPLACE, OP_REMOVE, OP_ONE_OFF, OP_PREFILL_DONE, OP_TERMINATE,
 OP_PIN, OP_UNPIN) = range(1, 11)
OPF_TOKENS_ON_DEVICE = 1
MAP_LOOKUP, MAP_ADMIT = 0, 1
IDS_ON_DEVICE = 1
KV_BF16, KV_FP16 = 0, 1
ROPE_INTERLEAVED, ATTN_FULL = 1, 1

EXPORTS = ("kvt_query_sizes", "kvt_create", "kvt_destroy", "kvt_apply_op", "kvt_map_blocks", "kvt_get_block_map",
           "kvt_classify", "kvt_get_states", "kvt_select_victims", "kvt_offload", "kvt_reload", "kvt_release",
           "kvt_compact", "kvt_copy_blocks", "kvt_hash_scratch_bytes", "kvt_hash_tokens", "kvt_get_stats",
           "kvt_last_error", "kvt_get_entries", "kvt_debug_load_resident", "kvt_set_profiling",
           "kvt_hash_tokens_noalloc", "kvt_debug_set_mover_variant", "kvt_exchange", "kvt_debug_set_lookup_variant", "kvt_move", "kvt_set_mover_ctas",
           "kvt_debug_set_wait_limit", "kvt_debug_set_classify_mode", "kvt_set_l2_residency", "kvt_debug_set_copy_delay",
           "kvt_append_kv", "kvt_attend", "kvt_attend_scratch_bytes", "kvt_set_tail_pool", "kvt_kv_check", "kvt_bound_keys",
           "kvt_select_blocks", "kvt_select_scratch_bytes", "kvt_attend_blocks", "kvt_weigh_blocks", "kvt_weigh_scratch_bytes",
           "kvt_evict_blocks")


class KvtError(RuntimeError):
    def __init__(self, code, what, detail=""):
        super().__init__(f"{what}: status {code} {detail}".strip())
        self.code = code


class Config(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("abi_version", "block_tokens", "n_layers", "n_kv_heads", "head_dim",
                                           "elem_bytes", "pool_layout", "n_hbm_blocks", "n_host_blocks",
                                           "table_capacity", "max_contexts", "max_messages", "max_batch_blocks",
                                           "policy_flags")] + \
               [("max_tokens", C.c_uint64), ("max_key_blocks", C.c_uint64), ("hash_seed", C.c_uint64),
                ("suspended_order", C.c_uint32), ("n_remote_blocks", C.c_uint32),
                ("hbm_pool", C.c_void_p), ("hbm_pool_bytes", C.c_uint64),
                ("host_pool", C.c_void_p), ("host_pool_bytes", C.c_uint64),
                ("dev_meta", C.c_void_p), ("dev_meta_bytes", C.c_uint64),
                ("dev_tokens", C.c_void_p), ("dev_tokens_bytes", C.c_uint64),
                ("remote_pool", C.c_void_p), ("remote_pool_bytes", C.c_uint64),
                ("stage_buf", C.c_void_p), ("stage_bytes", C.c_uint64)]


class Op(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("op", "ctx", "parent", "msg_start", "msg_end", "n_tokens", "flags",
                                           "reserved")] + [("tokens", C.c_void_p)]


class Batch(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("n_seqs", "n_tokens", "max_blocks", "max_q_len")] + \
               [("table_stride", C.c_uint64)] + [(n, C.c_void_p) for n in ("q_start", "kv_len", "block_table")]


class AppendArgs(C.Structure):
    _fields_ = [("b", Batch)] + [(n, C.c_uint32) for n in ("layer", "dtype", "n_q_heads", "flags", "rot_dim", "n_axes")] + \
               [(n, C.c_void_p) for n in ("q", "k", "v", "q_out")] + \
               [(n, C.c_uint64) for n in ("q_ts", "q_hs", "k_ts", "k_hs", "v_ts", "v_hs", "qo_ts", "qo_hs")] + \
               [(n, C.c_void_p) for n in ("freqs", "axis_of", "positions")] + [("pos_stride", C.c_uint64)]


class AttendArgs(C.Structure):
    _fields_ = [("b", Batch)] + [(n, C.c_uint32) for n in ("layer", "dtype", "n_q_heads", "flags", "window")] + \
               [("scale", C.c_float)] + [(n, C.c_void_p) for n in ("q", "out", "lse")] + \
               [(n, C.c_uint64) for n in ("q_ts", "q_hs", "o_ts", "o_hs")] + \
               [("scratch", C.c_void_p), ("scratch_bytes", C.c_uint64)]


class KeyBoundsArgs(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("exps", C.c_void_p), ("n_slots", C.c_uint64)]


class BoundArgs(C.Structure):
    _fields_ = [("b", Batch), ("layer", C.c_uint32), ("dtype", C.c_uint32), ("bounds", KeyBoundsArgs)]


class SelectArgs(C.Structure):
    _fields_ = [("b", Batch)] + [(n, C.c_uint32) for n in ("layer", "dtype", "n_q_heads", "n_blocks", "first", "last")] + \
               [("q", C.c_void_p), ("q_ts", C.c_uint64), ("q_hs", C.c_uint64), ("bounds", KeyBoundsArgs), ("out", C.c_void_p),
                ("scratch", C.c_void_p), ("scratch_bytes", C.c_uint64)]


class AttendBlocksArgs(C.Structure):
    _fields_ = [("b", Batch)] + [(n, C.c_uint32) for n in ("layer", "dtype", "n_q_heads", "n_blocks")] + \
               [("scale", C.c_float), ("reserved", C.c_uint32)] + [(n, C.c_void_p) for n in ("q", "out", "lse")] + \
               [(n, C.c_uint64) for n in ("q_ts", "q_hs", "o_ts", "o_hs")] + [("blocks", C.c_void_p)]


class WeighArgs(C.Structure):
    _fields_ = [("b", Batch)] + [(n, C.c_uint32) for n in ("layer", "dtype", "n_q_heads", "flags", "window")] + \
               [("scale", C.c_float), ("keep", C.c_float), ("reserved", C.c_uint32), ("q", C.c_void_p), ("lse", C.c_void_p),
                ("q_ts", C.c_uint64), ("q_hs", C.c_uint64), ("weights", C.c_void_p), ("out", C.c_void_p), ("w_stride", C.c_uint64),
                ("o_stride", C.c_uint64), ("scratch", C.c_void_p), ("scratch_bytes", C.c_uint64)]


class EvictArgs(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("n_seqs", "max_blocks", "n_blocks", "first", "last", "reserved")] + \
               [(n, C.c_void_p) for n in ("block_table", "kv_len", "weights")] + [("table_stride", C.c_uint64), ("w_stride", C.c_uint64)] + \
               [(n, C.c_void_p) for n in ("table_out", "kv_len_out", "weights_out", "evicted")] + \
               [(n, C.c_uint64) for n in ("table_out_stride", "w_out_stride", "evicted_stride")]


# the same layouts for struct.pack, which is what a call made thousands of times a second uses
_BATCH = "IIIIQPPP"
_APPEND = struct.Struct("@" + _BATCH + "IIIIIIPPPPQQQQQQQQPPPQ")
_ATTEND = struct.Struct("@" + _BATCH + "IIIIIfPPPQQQQPQ")
_FLT_MIN = 2.0 ** -126      # smallest scale that is told from 0

CALL_INFO_DTYPE = np.dtype([(n, np.uint32) for n in ("n_blocks", "hit_len", "n_hit_hbm", "n_hit_host",
                                                       "n_admissible", "n_admitted", "n_held", "n_pinned",
                                                       "n_hit_remote")])
STATS_FIELDS = ("clock", "n_contexts", "occ_hbm", "occ_host", "blocks_hashed", "hits_hbm", "hits_host", "misses",
                "inserted", "adopted", "dropped", "offloaded", "reloaded", "compacted", "bytes_d2h", "bytes_h2d",
                "bytes_d2d", "table_rebuilds", "tombstones", "kernel_launches", "mover_launches", "mover_ns",
                "mover_bytes", "lookup_ns", "lookup_blocks", "select_ns", "select_slots", "offloaded_clean",
                "blocks_rehashed", "occ_remote", "hits_remote", "demoted", "promoted", "classify_ns", "classify_items")

_lib = None


def load_library():
    """Loads libkvt.so (built in-tree by paper_2609_39819_b200.build). Raises if it is missing."""
    global _lib
    if _lib is None:
        if ALT_LIB:
            if not os.path.exists(ALT_LIB):
                raise RuntimeError(f"KVT_LIB={ALT_LIB} does not exist")
            lib_path = ALT_LIB
        else:
            lib_path = LIB_PATH
        try:                                       # a build step, not a fallback: (re)compile the CUDA library
            from . import build                    # in-tree when it is missing or older than its sources
            if not ALT_LIB:
                build.build_lib()
        except Exception as exc:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(f"{LIB_PATH} is missing and could not be built with nvcc ({exc}); "
                                   "there is no CPU fallback") from exc
            import warnings
            warnings.warn(f"libkvt.so could not be rebuilt ({exc}); loading the existing binary")
        lib = C.CDLL(lib_path)
        vp, u32, u64, i32 = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int32
        sig = {
            "kvt_query_sizes": [vp, vp, vp],
            "kvt_create": [vp, vp, vp],
            "kvt_destroy": [vp],
            "kvt_apply_op": [vp, vp, vp],
            "kvt_map_blocks": [vp, vp, u32, u32, vp, vp],
            "kvt_get_block_map": [vp, u32, vp, vp, vp, u32, vp, vp],
            "kvt_classify": [vp, vp],
            "kvt_get_states": [vp, u32, vp, u32, vp],
            "kvt_select_victims": [vp, u32, u32, u32, vp, vp, u32, vp, vp],
            "kvt_offload": [vp, vp, u32, vp, vp, vp],
            "kvt_reload": [vp, vp, u32, vp, vp],
            "kvt_exchange": [vp, vp, u32, vp, u32, vp, vp, vp, vp],
            "kvt_move": [vp, u32, u32, vp, u32, vp, vp, vp],
            "kvt_release": [vp, u32, vp, u32, vp],
            "kvt_compact": [vp, u32, vp, vp],
            "kvt_copy_blocks": [vp, u32, vp, u32, vp, u32, u32, vp],
            "kvt_hash_tokens": [vp, u64, u64, vp, vp, u64, vp],
            "kvt_hash_tokens_noalloc": [vp, u64, u64, vp, vp],
            "kvt_get_stats": [vp, vp],
            "kvt_last_error": [vp, vp, u32],
            "kvt_set_profiling": [vp, u32],
            "kvt_debug_set_mover_variant": [vp, u32],
            "kvt_debug_set_lookup_variant": [vp, u32],
            "kvt_set_mover_ctas": [vp, u32],
            "kvt_debug_set_wait_limit": [vp, u32],
            "kvt_debug_set_classify_mode": [vp, u32],
            "kvt_set_l2_residency": [vp, u32],
            "kvt_debug_set_copy_delay": [vp, u32],
            "kvt_get_entries": [vp, u32, vp, vp, vp, vp, vp, u32, vp],
            "kvt_debug_load_resident": [vp, vp, vp, vp, vp, vp, u32, u32, vp],
            "kvt_append_kv": [vp, vp, vp],
            "kvt_attend": [vp, vp, vp],
            "kvt_set_tail_pool": [vp, vp, u64],
            "kvt_kv_check": [vp, vp],
            "kvt_bound_keys": [vp, vp, vp],
            "kvt_select_blocks": [vp, vp, vp],
            "kvt_attend_blocks": [vp, vp, vp],
            "kvt_weigh_blocks": [vp, vp, vp],
            "kvt_evict_blocks": [vp, vp, vp],
        }
        for name, args in sig.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = i32
        lib.kvt_hash_scratch_bytes.argtypes = [u64]
        lib.kvt_hash_scratch_bytes.restype = u64
        for name in ("kvt_attend_scratch_bytes", "kvt_select_scratch_bytes", "kvt_weigh_scratch_bytes"):
            getattr(lib, name).argtypes = [vp, vp]
            getattr(lib, name).restype = u64
        _lib = lib
    return _lib


_native = None
_native_missing = None      # why there is none, once that is known


def load_native():
    """The native marshalling of append_kv and attend (built in-tree by build.build_torch_lib). Raises if it cannot be had."""
    global _native, _native_missing
    if _native is None:
        if _native_missing is not None:
            raise RuntimeError(_native_missing)
        import importlib.machinery
        import importlib.util
        import torch  # noqa: F401  (the module's symbols are torch's)
        from . import build
        try:
            # a binary older than its sources is not an answer: it may have other ideas of the library's structs
            loader = importlib.machinery.ExtensionFileLoader("_kvt_torch", build.build_torch_lib())
            module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_kvt_torch", loader))
            loader.exec_module(module)
        except Exception as exc:
            _native_missing = f"{build.TORCH_LIB} could not be built or loaded ({exc})"
            raise RuntimeError(_native_missing) from exc
        _native = module
    return _native


def _native_calls(lib):
    """append_kv and attend with native marshalling for `lib`; without it functions that leave every call to the marshalling in
    Python, which takes 4 us longer and does the same."""
    try:
        native = load_native()
    except RuntimeError as exc:
        import warnings
        warnings.warn(f"append_kv and attend marshal their arguments in Python: {exc}")
        return (lambda *args: NotImplemented,) * 2
    entry = lambda f: C.cast(f, C.c_void_p).value      # noqa: E731
    return (functools.partial(native.append, entry(lib.kvt_append_kv)),
            functools.partial(native.attend, entry(lib.kvt_attend), entry(lib.kvt_attend_scratch_bytes)))


def _native_block_calls(lib):
    """The same for bound_keys, select_blocks, attend_blocks, weigh_blocks and evict_blocks."""
    try:
        native = load_native()
    except RuntimeError:        # _native_calls has said so
        return (lambda *args: NotImplemented,) * 5
    entry = lambda f: C.cast(f, C.c_void_p).value      # noqa: E731
    return (functools.partial(native.bound, entry(lib.kvt_bound_keys)),
            functools.partial(native.select, entry(lib.kvt_select_blocks), entry(lib.kvt_select_scratch_bytes)),
            functools.partial(native.attend_blocks, entry(lib.kvt_attend_blocks)),
            functools.partial(native.weigh, entry(lib.kvt_weigh_blocks), entry(lib.kvt_weigh_scratch_bytes)),
            functools.partial(native.evict, entry(lib.kvt_evict_blocks)))


def _p(a):
    return a.ctypes.data_as(C.c_void_p) if a is not None else None


def _u32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.uint32))


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def hash_tokens(tokens_dev, seed: int = 0):
    """Chained block keys of a device token tensor (int32/uint32 view, 16-byte aligned) -> int64 tensor
    whose bit patterns are the unsigned 64-bit keys."""
    import torch
    lib = load_library()
    n = tokens_dev.numel()
    keys = torch.empty(n // 16, dtype=torch.int64, device=tokens_dev.device)
    sb = lib.kvt_hash_scratch_bytes(n)
    scratch = torch.empty(sb, dtype=torch.uint8, device=tokens_dev.device)
    rc = lib.kvt_hash_tokens(tokens_dev.data_ptr(), n, seed, keys.data_ptr(), scratch.data_ptr(), sb, _stream())
    if rc:
        raise KvtError(rc, "hash_tokens")
    return keys


HASH_NOALLOC_MAX_TOKENS = 1 << 22


def hash_tokens_noalloc(tokens_dev, keys_out, seed: int = 0) -> int:
    """Block keys of a device token tensor written into the caller's `keys_out` (int64, >= n // 16
    elements) with the library's built-in scratch: for callers that must not allocate. Returns the
    status code (KVT_E_NOSPACE beyond HASH_NOALLOC_MAX_TOKENS)."""
    lib = load_library()
    return lib.kvt_hash_tokens_noalloc(tokens_dev.data_ptr(), tokens_dev.numel(), seed, keys_out.data_ptr(), _stream())


class Rope:
    """The rotation `Engine.append_kv` applies: pair j of the leading `rot_dim` elements of a head turns by
    position * freqs[j] radians. Frequencies are theta ** (-2 j / rot_dim) unless `freqs` (rot_dim / 2 numbers) gives
    others. `sections` shares the pairs out among several position axes (time, height, width): so many consecutive
    pairs per axis, adding up to rot_dim / 2; `axis_of` names the axis of each pair instead. `interleaved`: pairs are
    neighbours (2j, 2j + 1); otherwise (j, j + rot_dim / 2)."""

    def __init__(self, rot_dim, theta=10000.0, sections=None, axis_of=None, interleaved=False, freqs=None, device="cuda"):
        import torch
        if rot_dim < 0 or rot_dim % 2:
            raise ValueError("Rope: rot_dim must be even")
        half = rot_dim // 2
        if freqs is None:
            freqs = [theta ** (-2.0 * j / rot_dim) for j in range(half)]
        if len(freqs) != half:
            raise ValueError(f"Rope: {half} frequencies expected, got {len(freqs)}")
        if sections is not None:
            if axis_of is not None or any(n < 0 for n in sections) or sum(sections) != half:
                raise ValueError(f"Rope: sections must add up to {half}, without axis_of")
            axis_of = [i for i, n in enumerate(sections) for _ in range(n)]
        self.rot_dim, self.interleaved = rot_dim, bool(interleaved)
        self.freqs = torch.as_tensor(freqs, dtype=torch.float64).to(device).contiguous()
        self.n_axes, self.axis_of = 1, None
        if axis_of is not None:
            axis_of = [int(x) for x in axis_of]
            if len(axis_of) != half or any(not 0 <= x < 256 for x in axis_of):
                raise ValueError(f"Rope: axis_of needs {half} axes below 256")
            self.n_axes = len(sections) if sections is not None else max(axis_of, default=0) + 1
            self.axis_of = torch.tensor(axis_of, dtype=torch.uint8).to(device)


class KeyBounds:
    """Bounds of the keys of an engine's full blocks (`Engine.key_bounds` makes them, `Engine.bound_keys` fills them in): int8 codes
    [layers, slots, KV heads, 2, width] and uint8 exps [layers, slots, KV heads]. In channel d the keys of a block are at most
    codes[l, s, h, 0, d] * 2 ** (exps[l, s, h] - 127) and at least -codes[l, s, h, 1, d] * 2 ** (...). dtype: that of the pool's
    elements."""

    def __init__(self, dtype, codes, exps):
        self.dtype, self.codes, self.exps = dtype, codes, exps


class Engine:
    """One cache engine on the current CUDA device. Allocates the pools and arenas with torch and
    hands raw pointers to the library."""

    def __init__(self, n_layers, n_kv_heads, head_dim, elem_bytes=2, pool_layout=LAYOUT_LAYER_MAJOR,
                 n_hbm_blocks=128, n_host_blocks=512, max_contexts=64, hash_seed=0, suspended_order=ORDER_MRU,
                 metadata_only=False, table_capacity=None, max_messages=1 << 16, max_batch_blocks=None,
                 max_tokens=1 << 22, max_key_blocks=None, host_pool_on_device=False, zero_pools=True, policy_flags=0,
                 n_remote_blocks=0, stage_mib=256, device="cuda", n_tail_blocks=0):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2609_39819_b200 needs a CUDA device (there is no CPU fallback)")
        self.torch = torch
        self.L = load_library()
        self.device = torch.device(device)
        self.n_layers, self.n_kv_heads, self.head_dim, self.elem_bytes = n_layers, n_kv_heads, head_dim, elem_bytes
        self.pool_layout = pool_layout
        self.n_hbm_blocks, self.n_host_blocks, self.n_remote_blocks = n_hbm_blocks, n_host_blocks, n_remote_blocks
        self.chunk_bytes = 16 * n_kv_heads * head_dim * elem_bytes
        self.n_chunks = 2 * n_layers
        self.block_bytes = self.chunk_bytes * self.n_chunks
        self.metadata_only = metadata_only
        n_total = n_hbm_blocks + n_host_blocks + n_remote_blocks
        if table_capacity is None:
            table_capacity = 1 << max(4, (2 * n_total - 1).bit_length())
        if max_batch_blocks is None:
            max_batch_blocks = max(max_tokens // 16, 1)
        if max_key_blocks is None:
            max_key_blocks = max(max_tokens // 8, 64)
        cfg = Config()
        cfg.abi_version, cfg.block_tokens = 3, 16
        cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, cfg.elem_bytes = n_layers, n_kv_heads, head_dim, elem_bytes
        cfg.pool_layout, cfg.n_hbm_blocks, cfg.n_host_blocks = pool_layout, n_hbm_blocks, n_host_blocks
        cfg.n_remote_blocks = n_remote_blocks
        cfg.table_capacity, cfg.max_contexts, cfg.max_messages = table_capacity, max_contexts, max_messages
        cfg.max_batch_blocks, cfg.max_tokens, cfg.max_key_blocks = max_batch_blocks, max_tokens, max_key_blocks
        cfg.hash_seed, cfg.suspended_order, cfg.policy_flags = hash_seed, suspended_order, policy_flags
        mb, tb = C.c_uint64(0), C.c_uint64(0)
        rc = self.L.kvt_query_sizes(C.byref(cfg), C.byref(mb), C.byref(tb))
        if rc:
            raise KvtError(rc, "query_sizes")
        self.meta = torch.empty(mb.value + 256, dtype=torch.uint8, device=self.device)
        self.tokens = torch.empty(tb.value + 256, dtype=torch.uint8, device=self.device)
        cfg.dev_meta, cfg.dev_meta_bytes = self._align(self.meta), mb.value
        cfg.dev_tokens, cfg.dev_tokens_bytes = self._align(self.tokens), tb.value
        if metadata_only:
            self.hbm_pool = self.host_pool = self.remote_pool = None
        else:
            new = torch.zeros if zero_pools else torch.empty
            self.hbm_pool = new(n_hbm_blocks * self.block_bytes, dtype=torch.uint8, device=self.device)
            nh = max(n_host_blocks, 1) * self.block_bytes
            if host_pool_on_device:   # second tier kept in HBM (in-device measurements)
                self.host_pool = new(nh, dtype=torch.uint8, device=self.device)
            else:
                self.host_pool = new(nh, dtype=torch.uint8, pin_memory=True)
            cfg.hbm_pool, cfg.hbm_pool_bytes = self.hbm_pool.data_ptr(), self.hbm_pool.numel()
            cfg.host_pool, cfg.host_pool_bytes = self.host_pool.data_ptr(), self.host_pool.numel()
            # the remote tier is stood in for by one more buffer of the same kind as the host tier
            nr = max(n_remote_blocks, 1) * self.block_bytes
            if host_pool_on_device:
                self.remote_pool = new(nr, dtype=torch.uint8, device=self.device)
            else:
                self.remote_pool = new(nr, dtype=torch.uint8, pin_memory=True)
            if n_remote_blocks:
                cfg.remote_pool, cfg.remote_pool_bytes = self.remote_pool.data_ptr(), self.remote_pool.numel()
            # staging ring for copy-engine transfers between HBM and a host-memory tier (large blocks only)
            self.stage_buf = None
            if stage_mib and not host_pool_on_device and (n_host_blocks or n_remote_blocks):
                self.stage_buf = torch.empty(stage_mib << 20, dtype=torch.uint8, device=self.device)
                cfg.stage_buf, cfg.stage_bytes = self.stage_buf.data_ptr(), self.stage_buf.numel()
        self.cfg = cfg
        h = C.c_void_p()
        rc = self.L.kvt_create(C.byref(cfg), _stream(), C.byref(h))
        if rc:
            raise KvtError(rc, "create")
        self.h = h
        self._dev = self.meta.device
        self._dev_index = self._dev.index
        self._kv_dtypes = {torch.bfloat16: KV_BF16, torch.float16: KV_FP16}
        # the address of the device's current stream, without a Stream object around it (2 us of a call of 10)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda index: torch.cuda.current_stream(index).cuda_stream)
        self._append_native, self._attend_native = _native_calls(self.L)
        self._bound_native, self._select_native, self._attend_blocks_native, self._weigh_native, self._evict_native = \
            _native_block_calls(self.L)
        self.tail_pool = None
        if n_tail_blocks:       # blocks outside every tier: slot ids n_hbm_blocks + i of append_kv and attend
            self.set_tail_pool((torch.zeros if zero_pools else torch.empty)(n_tail_blocks * self.block_bytes, dtype=torch.uint8,
                                                                            device=self.device))

    @staticmethod
    def _align(t):
        return (t.data_ptr() + 255) // 256 * 256

    def close(self):
        if getattr(self, "h", None):
            self.L.kvt_destroy(self.h)
            self.h = None
            self.hbm_pool = self.host_pool = self.remote_pool = self.meta = self.tokens = self.stage_buf = self.tail_pool = None   # release the memory

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_profiling(self, on=True):
        self._check(self.L.kvt_set_profiling(self.h, 1 if on else 0), "set_profiling")

    def set_mover_variant(self, variant):
        self._check(self.L.kvt_debug_set_mover_variant(self.h, variant), "set_mover_variant")

    def set_mover_ctas(self, max_ctas):
        self._check(self.L.kvt_set_mover_ctas(self.h, max_ctas), "set_mover_ctas")

    def set_lookup_variant(self, variant):
        self._check(self.L.kvt_debug_set_lookup_variant(self.h, variant), "set_lookup_variant")

    def set_copy_delay(self, delay_ns):
        self._check(self.L.kvt_debug_set_copy_delay(self.h, int(delay_ns)), "set_copy_delay")

    def set_l2_residency(self, on=True):
        self._check(self.L.kvt_set_l2_residency(self.h, 1 if on else 0), "set_l2_residency")

    def set_classify_mode(self, mode):
        self._check(self.L.kvt_debug_set_classify_mode(self.h, mode), "set_classify_mode")

    def set_wait_limit(self, polls):
        self._check(self.L.kvt_debug_set_wait_limit(self.h, polls), "set_wait_limit")

    def last_error(self):
        buf = C.create_string_buffer(256)
        self.L.kvt_last_error(self.h, buf, 256)
        return buf.value.decode()

    def _check(self, rc, what):
        if rc:
            raise KvtError(rc, what, self.last_error())

    # ---- primitives ---------------------------------------------------------------------------
    def apply_op_rc(self, op, ctx, parent=0, msg_start=0, msg_end=0, tokens=None) -> int:
        flags, ptr, n = 0, None, 0
        keep = None
        if tokens is not None:
            if hasattr(tokens, "data_ptr"):      # torch tensor: device memory, or (pinned) host memory
                keep = tokens
                flags, ptr, n = (OPF_TOKENS_ON_DEVICE if tokens.is_cuda else 0), tokens.data_ptr(), tokens.numel()
            else:
                keep = _u32(tokens)
                ptr, n = keep.ctypes.data, len(keep)
        o = Op(op, ctx, parent, msg_start, msg_end, n, flags, 0, ptr)
        return self.L.kvt_apply_op(self.h, C.byref(o), _stream())

    def _op(self, what, *a, **k):
        self._check(self.apply_op_rc(*a, **k), what)

    def spawn(self, ctx): self._op("spawn", OP_SPAWN, ctx)
    def fork(self, parent, child, end): self._op("fork", OP_FORK, child, parent=parent, msg_end=end)
    def append(self, ctx, tokens): self._op("append", OP_APPEND, ctx, tokens=tokens)
    def replace(self, ctx, s, e, tokens): self._op("replace", OP_REPLACE, ctx, msg_start=s, msg_end=e, tokens=tokens)
    def remove(self, ctx, s, e): self._op("remove", OP_REMOVE, ctx, msg_start=s, msg_end=e)

    def one_off(self, ctx, s=0, e=None):
        self._op("one_off", OP_ONE_OFF, ctx, msg_start=s, msg_end=0xFFFFFFFF if e is None else e)

    def pin(self, ctx, s, e): self._op("pin", OP_PIN, ctx, msg_start=s, msg_end=e)
    def unpin(self, ctx, s, e): self._op("unpin", OP_UNPIN, ctx, msg_start=s, msg_end=e)
    def prefill_done(self, ctx): self._op("prefill_done", OP_PREFILL_DONE, ctx)
    def terminate(self, ctx): self._op("terminate", OP_TERMINATE, ctx)

    # ---- hash / lookup / admit ---------------------------------------------------------------
    def map_blocks_rc(self, ctx_ids, phase):
        ids = _u32(ctx_ids)
        out = np.zeros(len(ids), dtype=CALL_INFO_DTYPE)
        rc = self.L.kvt_map_blocks(self.h, _p(ids), len(ids), phase, _p(out), _stream())
        return rc, out

    def map_blocks(self, ctx_ids, phase):
        rc, out = self.map_blocks_rc(ctx_ids, phase)
        self._check(rc, "map_blocks")
        return out

    def get_block_map(self, ctx):
        n = C.c_uint32(0)
        rc = self.L.kvt_get_block_map(self.h, ctx, None, None, None, 0, C.byref(n), _stream())
        if rc not in (OK, E_BUFSZ):
            self._check(rc, "get_block_map")
        nb = n.value
        keys = np.empty(nb, np.uint64); tier = np.empty(nb, np.uint8); slot = np.empty(nb, np.uint32)
        self._check(self.L.kvt_get_block_map(self.h, ctx, _p(keys), _p(tier), _p(slot), nb, C.byref(n), _stream()),
                    "get_block_map")
        return keys, tier, slot

    # ---- classify / select ----------------------------------------------------------------------
    def classify(self):
        self._check(self.L.kvt_classify(self.h, _stream()), "classify")

    def _tier_size(self, tier):
        sizes = (self.n_hbm_blocks, self.n_host_blocks, self.n_remote_blocks)
        return sizes[tier] if 0 <= tier < 3 else 0      # an unknown tier is for the library to reject

    def get_states(self, tier):
        st = np.zeros(self._tier_size(tier), np.uint8)
        self._check(self.L.kvt_get_states(self.h, tier, _p(st), len(st), _stream()), "get_states")
        return st

    def victim_buffers(self, n):
        """A pair of pinned host arrays (slots, states) for `out=` of select_victims: the selection's last kernel
        writes the list straight into them instead of staging it for a CPU copy."""
        import torch
        ts = torch.empty(n, dtype=torch.int32, pin_memory=True); tt = torch.empty(n, dtype=torch.uint8, pin_memory=True)
        self._victim_bufs = getattr(self, "_victim_bufs", []) + [(ts, tt)]     # the arrays below do not own the memory
        return ts.numpy().view(np.uint32), tt.numpy()

    def select_victims(self, tier, n_req, include_pinned=False, out=None):
        cap = min(n_req, self._tier_size(tier))
        if out is None:
            slots = np.empty(cap, np.uint32); states = np.empty(cap, np.uint8)     # filled by the call up to n
        else:
            slots, states = out
            if len(slots) < cap or len(states) < cap or slots.dtype != np.uint32 or states.dtype != np.uint8:
                raise ValueError("select_victims: out arrays too small or of the wrong type")
        n = C.c_uint32(0)
        self._check(self.L.kvt_select_victims(self.h, tier, n_req, 1 if include_pinned else 0, _p(slots), _p(states),
                                              cap, C.byref(n), _stream()), "select_victims")
        return slots[:n.value], states[:n.value]

    # ---- movement -------------------------------------------------------------------------------
    def offload(self, slots):
        s = _u32(slots); nd = C.c_uint32(0); nx = C.c_uint32(0)
        rc = self.L.kvt_offload(self.h, _p(s), len(s), C.byref(nd), C.byref(nx), _stream())
        return rc, nd.value, nx.value

    def reload(self, slots):
        s = _u32(slots); nd = C.c_uint32(0)
        rc = self.L.kvt_reload(self.h, _p(s), len(s), C.byref(nd), _stream())
        return rc, nd.value

    def move(self, src_tier, dst_tier, slots):
        s = _u32(slots)
        nd, nx = C.c_uint32(0), C.c_uint32(0)
        rc = self.L.kvt_move(self.h, src_tier, dst_tier, _p(s), len(s), C.byref(nd), C.byref(nx), _stream())
        return rc, nd.value, nx.value

    def exchange(self, out_slots, in_slots):
        o, i = _u32(out_slots), _u32(in_slots)
        a, b, c = C.c_uint32(0), C.c_uint32(0), C.c_uint32(0)
        rc = self.L.kvt_exchange(self.h, _p(o), len(o), _p(i), len(i), C.byref(a), C.byref(b), C.byref(c), _stream())
        return rc, a.value, b.value, c.value

    def release_rc(self, tier, slots):
        s = _u32(slots)
        return self.L.kvt_release(self.h, tier, _p(s), len(s), _stream())

    def release(self, tier, slots):
        self._check(self.release_rc(tier, slots), "release")

    def compact(self, tier):
        n = C.c_uint32(0)
        self._check(self.L.kvt_compact(self.h, tier, C.byref(n), _stream()), "compact")
        return n.value

    def copy_blocks(self, src_tier, src, dst_tier, dst):
        """src / dst: host sequences, or device int32 tensors (ids stay on the device)."""
        if hasattr(src, "data_ptr"):
            rc = self.L.kvt_copy_blocks(self.h, src_tier, src.data_ptr(), dst_tier, dst.data_ptr(), src.numel(),
                                        IDS_ON_DEVICE, _stream())
        else:
            s, d = _u32(src), _u32(dst)
            rc = self.L.kvt_copy_blocks(self.h, src_tier, _p(s), dst_tier, _p(d), len(s), 0, _stream())
        self._check(rc, "copy_blocks")

    # ---- model-side operators on the HBM pool -----------------------------------------------------
    def set_tail_pool(self, pool):
        """Tail blocks (slot ids n_hbm_blocks + i): a uint8 device tensor of whole blocks, block-major; None removes it. Calls made
        or captured before keep the tensor they were given, which has to be kept alive as long as they may run."""
        if pool is not None and (pool.device != self._dev or pool.dtype != self.torch.uint8 or not pool.is_contiguous()):
            raise ValueError(f"set_tail_pool: a contiguous uint8 tensor on the engine's device ({self._dev}) expected")
        self._check(self.L.kvt_set_tail_pool(self.h, pool.data_ptr() if pool is not None else None,
                                             pool.numel() if pool is not None else 0), "set_tail_pool")
        self.tail_pool = pool

    def _kv_dtype(self, x, what):
        code = self._kv_dtypes.get(x.dtype)
        if code is None:
            raise ValueError(f"{what}: bfloat16 or float16 expected, got {x.dtype}")
        return code

    def _kv_tensor(self, x, what, shape, dtype):
        """(address, token stride, head stride) of a [tokens, heads, head_dim] tensor."""
        if x.dtype is not dtype or x.shape != shape or x.get_device() != self._dev_index:
            raise ValueError(f"{what}: {dtype} tensor {tuple(shape)} on {self._dev} expected, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        if x.requires_grad and self.torch.is_grad_enabled():
            raise ValueError(f"{what}: the tensor requires a gradient, and there is no backward pass; call under torch.no_grad()")
        ts, hs, es = x.stride()
        if es != 1 and shape[2] > 1:
            raise ValueError(f"{what}: the elements of a head must be consecutive")
        return x.data_ptr(), ts, hs

    def _kv_batch(self, what, n_tokens, block_table, q_start, kv_len, max_q_len):
        i32, dev = self.torch.int32, self._dev_index
        if block_table.dtype is not i32 or q_start.dtype is not i32 or kv_len.dtype is not i32 or \
                block_table.dim() != 2 or q_start.dim() != 1 or kv_len.dim() != 1:
            raise ValueError(f"{what}: block_table [sequences, blocks], q_start and kv_len must be int32")
        n, m = block_table.shape
        ts, es = block_table.stride()
        if kv_len.numel() != n or q_start.numel() != n + 1 or (es != 1 and m > 1) or not q_start.is_contiguous() or \
                not kv_len.is_contiguous():
            raise ValueError(f"{what}: {n} table rows need {n} lengths and {n + 1} starts, with consecutive elements")
        if block_table.get_device() != dev or q_start.get_device() != dev or kv_len.get_device() != dev:
            raise ValueError(f"{what}: block_table, q_start and kv_len must be on {self._dev}")
        return n, n_tokens, m, max_q_len or 0, ts, q_start.data_ptr(), kv_len.data_ptr(), block_table.data_ptr()

    def _kv_stream(self):
        return self._raw_stream(self._dev_index)

    def append_kv(self, layer, k, v, block_table, q_start, kv_len, rope=None, positions=None, q=None, q_out=None):
        """Writes the new tokens' keys (rotated) and values into the blocks of `layer` and returns the rotated queries
        (in `q_out`, which may be `q`, or a new tensor; None without q). k, v: [tokens, n_kv_heads, head_dim], q:
        [tokens, heads, head_dim], bf16 or fp16, any strides with consecutive elements. Sequence s brings rows
        [q_start[s], q_start[s+1]) and holds kv_len[s] tokens with them; block_table[s, b] is the slot of its b-th
        16-token block (below n_hbm_blocks: HBM tier; above: tail block). positions: int32 [tokens] or [axes, tokens],
        by default the tokens' indices in their sequences. Asynchronous on the current stream; ids and lengths outside
        their ranges are skipped and reported by kv_check(). No backward pass: tensors that require gradients are taken
        under torch.no_grad() only."""
        done = self._append_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                                   layer, k, v, block_table, q_start, kv_len,
                                   *((0, 1, None, None, False) if rope is None else
                                     (rope.rot_dim, rope.n_axes, rope.freqs, rope.axis_of, rope.interleaved)), positions, q, q_out)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "append_kv")
            return done
        # something is not as it should be (what, is said here), or only of another type than it might be
        torch = self.torch
        if layer < 0:
            raise ValueError("append_kv: layer cannot be negative")
        dt = self._kv_dtype(k, "append_kv")
        t, h, d = k.shape[0], self.n_kv_heads, self.head_dim
        kp, kts, khs = self._kv_tensor(k, "append_kv: k", (t, h, d), k.dtype)
        vp, vts, vhs = self._kv_tensor(v, "append_kv: v", (t, h, d), k.dtype)
        batch = self._kv_batch("append_kv", t, block_table, q_start, kv_len, 0)
        hq = qp = qts = qhs = op = ots = ohs = 0
        if q is not None:
            hq = q.shape[1] if q.dim() == 3 else 0
            qp, qts, qhs = self._kv_tensor(q, "append_kv: q", (t, hq, d), k.dtype)
            if q_out is None:
                q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
                op, ots, ohs = q_out.data_ptr(), hq * d, d
            else:
                op, ots, ohs = self._kv_tensor(q_out, "append_kv: q_out", (t, hq, d), k.dtype)
                if (ots == 0 and t > 1) or (ohs == 0 and hq > 1):
                    raise ValueError("append_kv: q_out is a broadcast tensor")
                if qp == op and (qts, qhs) != (ots, ohs):
                    raise ValueError("append_kv: q_out in the place of q needs its strides")
        elif q_out is not None:
            raise ValueError("append_kv: q_out without q")
        rot = flags = freqs = axis_of = pos = pos_stride = 0
        n_axes = 1
        if rope is not None:
            rot, n_axes, freqs = rope.rot_dim, rope.n_axes, rope.freqs.data_ptr()
            if rope.freqs.get_device() != self._dev_index:
                raise ValueError(f"append_kv: rope is on {rope.freqs.device}, the engine on {self._dev}")
            if rope.interleaved:
                flags = ROPE_INTERLEAVED
            if rope.axis_of is not None:
                axis_of = rope.axis_of.data_ptr()
            if positions is None and n_axes > 1:
                raise ValueError(f"append_kv: {n_axes} axes need positions")
        if positions is not None:
            p2 = positions if positions.dim() == 2 else positions[None]
            if rope is None or p2.dtype != torch.int32 or p2.shape != (n_axes, t) or p2.get_device() != self._dev_index or \
                    (t > 1 and p2.stride(1) != 1):
                raise ValueError(f"append_kv: positions must be int32 [{n_axes}, {t}] on {self._dev}, with a rope")
            pos, pos_stride = p2.data_ptr(), p2.stride(0)
        a = _APPEND.pack(*batch, layer, dt, hq, flags, rot, n_axes, qp, kp, vp, op, qts, qhs, kts, khs, vts, vhs, ots, ohs,
                         freqs, axis_of, pos, pos_stride)
        self._check(self.L.kvt_append_kv(self.h, a, self._kv_stream()), "append_kv")
        return q_out

    def attend(self, layer, q, block_table, q_start, kv_len, max_q_len=None, causal=True, window=None, scale=None, out=None,
               lse=None):
        """softmax(scale q k^T) v of the new tokens' queries over everything their sequences hold in `layer` (append
        first: the new tokens are among the kv_len[s]). q: [tokens, heads, head_dim], heads a multiple of n_kv_heads;
        batch as in append_kv. causal: a query sees the keys up to its own, with `window` the last `window` of them;
        causal=False: all kv_len keys. scale: 1 / sqrt(head_dim) if None. max_q_len: most new tokens of one sequence,
        if known (chooses the kernel; results agree within their rounding). out, lse ([tokens, heads] float32, contiguous): written if
        given; rows behind the last sequence stay as they are. Returns out. Asynchronous on the current stream. No backward
        pass: tensors that require gradients are taken under torch.no_grad() only."""
        done = self._attend_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                                   layer, q, block_table, q_start, kv_len, max_q_len, causal, window, scale, out, lse)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "attend")
            return done
        # something is not as it should be (what, is said here), or only of another type than it might be
        torch = self.torch
        if layer < 0 or (max_q_len or 0) < 0 or (window or 0) < 0:
            raise ValueError("attend: layer, max_q_len and window cannot be negative")
        dt = self._kv_dtype(q, "attend")
        t, hq, d = q.shape if q.dim() == 3 else (0, 0, 0)
        qp, qts, qhs = self._kv_tensor(q, "attend: q", (t, hq, self.head_dim), q.dtype)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            op, ots, ohs = out.data_ptr(), hq * d, d
        else:
            op, ots, ohs = self._kv_tensor(out, "attend: out", (t, hq, d), q.dtype)
            if (ots == 0 and t > 1) or (ohs == 0 and hq > 1):
                raise ValueError("attend: out is a broadcast tensor")
        if lse is not None and (lse.dtype != torch.float32 or lse.shape != (t, hq) or lse.get_device() != self._dev_index or
                                not lse.is_contiguous()):
            raise ValueError(f"attend: lse must be a contiguous float32 [{t}, {hq}] tensor on {self._dev}")
        if lse is not None and lse.requires_grad and torch.is_grad_enabled():
            raise ValueError("attend: lse requires a gradient, and there is no backward pass; call under torch.no_grad()")
        batch = self._kv_batch("attend", t, block_table, q_start, kv_len, max_q_len)
        flags, lsep = 0 if causal else ATTN_FULL, lse.data_ptr() if lse is not None else 0
        # 0, which is the library's word for the default, becomes next to 0
        factor = 0.0 if scale is None else max(float(scale), _FLT_MIN) if scale >= 0 else float(scale)
        probe = _ATTEND.pack(*batch, layer, dt, hq, flags, window or 0, factor, qp, op, lsep, qts, qhs, ots, ohs, 0, 0)
        n = self.L.kvt_attend_scratch_bytes(self.h, probe)
        # from the current stream's pool, or the capture's: nobody else has it while this call's kernels run
        scratch = torch.empty(n, dtype=torch.uint8, device=self._dev) if n else None
        a = _ATTEND.pack(*batch, layer, dt, hq, flags, window or 0, factor, qp, op, lsep, qts, qhs, ots, ohs,
                         scratch.data_ptr() if n else 0, n)
        self._check(self.L.kvt_attend(self.h, a, self._kv_stream()), "attend")
        return out

    # ---- choosing blocks ----------------------------------------------------------------------------
    def key_bounds(self, dtype):
        """Room for the bounds of all blocks in the HBM pool and the tail pool of now, for bound_keys and select_blocks. dtype: of
        the pool's elements, bfloat16 or float16."""
        torch = self.torch
        if self.metadata_only or dtype not in self._kv_dtypes or self.elem_bytes != 2:
            raise ValueError("key_bounds: a pool of bfloat16 or float16 elements expected")
        n = self.n_hbm_blocks + (self.tail_pool.numel() // self.block_bytes if self.tail_pool is not None else 0)
        shape = (self.n_layers, n, self.n_kv_heads)
        return KeyBounds(dtype, torch.zeros(*shape, 2, (self.head_dim + 15) // 16 * 16, dtype=torch.int8, device=self._dev),
                         torch.zeros(shape, dtype=torch.uint8, device=self._dev))

    def _bounds(self, what, bounds):
        torch = self.torch
        codes, exps = bounds.codes, bounds.exps
        n = codes.shape[1] if codes.dim() == 5 else 0
        shape = (self.n_layers, n, self.n_kv_heads)
        if codes.shape != (*shape, 2, (self.head_dim + 15) // 16 * 16) or exps.shape != shape or codes.dtype is not torch.int8 or \
                exps.dtype is not torch.uint8 or not codes.is_contiguous() or not exps.is_contiguous() or \
                codes.get_device() != self._dev_index or exps.get_device() != self._dev_index:
            raise ValueError(f"{what}: bounds are not this engine's (key_bounds() makes them)")
        return KeyBoundsArgs(codes.data_ptr(), exps.data_ptr(), n)

    def _kv_lse(self, what, lse, t, hq):
        if lse.dtype is not self.torch.float32 or lse.shape != (t, hq) or lse.get_device() != self._dev_index or not lse.is_contiguous():
            raise ValueError(f"{what}: lse must be a contiguous float32 [{t}, {hq}] tensor on {self._dev}")
        if lse.requires_grad and self.torch.is_grad_enabled():
            raise ValueError(f"{what}: lse requires a gradient, and there is no backward pass; call under torch.no_grad()")
        return lse.data_ptr()

    def _kv_scale(self, scale):
        # 0, which is the library's word for the default, becomes next to 0
        return 0.0 if scale is None else max(float(scale), _FLT_MIN) if scale >= 0 else float(scale)

    def _kv_rows(self, what, x, dtype, shape):
        """(address, row stride) of a table [rows, elements]."""
        if x.dtype is not dtype or x.shape != shape or x.get_device() != self._dev_index or (shape[1] > 1 and x.stride(1) != 1):
            raise ValueError(f"{what}: {dtype} tensor {tuple(shape)} on {self._dev} with consecutive elements expected, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        if x.requires_grad and self.torch.is_grad_enabled():
            raise ValueError(f"{what}: the tensor requires a gradient, and there is no backward pass; call under torch.no_grad()")
        return x.data_ptr(), x.stride(0)

    def bound_keys(self, layer, bounds, block_table, q_start, kv_len, n_tokens):
        """Writes the bounds of the blocks of `layer` that the batch's new tokens fill, from the keys in the pool: call it behind
        append_kv with the same batch; n_tokens: rows of that batch. After blocks have come into their slots in another way
        (reload, a prefix that was there), a batch that counts their tokens as new makes their bounds. Asynchronous on the current
        stream."""
        done = self._bound_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                                  self.n_layers, layer, self._kv_dtypes.get(bounds.dtype), bounds.codes, bounds.exps, block_table, q_start,
                                  kv_len, n_tokens)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "bound_keys")
            return None
        # something is not as it should be (what, is said here), or only of another type than it might be
        if layer < 0 or n_tokens < 0:
            raise ValueError("bound_keys: layer and n_tokens cannot be negative")
        batch = self._kv_batch("bound_keys", n_tokens, block_table, q_start, kv_len, 0)
        a = BoundArgs(Batch(*batch), layer, self._kv_dtypes[bounds.dtype], self._bounds("bound_keys", bounds))
        self._check(self.L.kvt_bound_keys(self.h, C.byref(a), self._kv_stream()), "bound_keys")

    def select_blocks(self, layer, q, bounds, block_table, q_start, kv_len, n_blocks, first=1, last=2, max_q_len=None, out=None):
        """For each new token and KV head the numbers of the n_blocks blocks of its sequence that its queries are to attend to: int32
        [tokens, KV heads, n_blocks], ascending, -1 behind the last. Always among them: the first `first` blocks and the `last` last up
        to the token's own; the others are those of the largest scores by `bounds` (include/kvt.h says how they are reckoned; they are
        exact, so that neither the batch nor the kernel has a say). q: rotated queries, batch as in attend (max_q_len is taken and has no
        effect); rows behind the last sequence stay as they are. Asynchronous on the current stream."""
        done = self._select_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                                   self.n_layers, layer, self._kv_dtypes.get(bounds.dtype), q, bounds.codes, bounds.exps, block_table,
                                   q_start, kv_len, n_blocks, first, last, max_q_len, out)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "select_blocks")
            return done
        # something is not as it should be (what, is said here), or only of another type than it might be
        torch = self.torch
        if layer < 0 or (max_q_len or 0) < 0 or min(first, last, n_blocks) < 0:
            raise ValueError("select_blocks: layer, max_q_len, first, last and n_blocks cannot be negative")
        dt = self._kv_dtype(q, "select_blocks")
        if q.dtype != bounds.dtype:
            raise ValueError(f"select_blocks: q is {q.dtype}, the bounds are of {bounds.dtype} keys")
        t, hq, d = q.shape if q.dim() == 3 else (0, 0, 0)
        qp, qts, qhs = self._kv_tensor(q, "select_blocks: q", (t, hq, self.head_dim), q.dtype)
        shape = (t, self.n_kv_heads, n_blocks)
        if out is None:
            out = torch.empty(shape, dtype=torch.int32, device=self._dev)
        elif out.dtype is not torch.int32 or out.shape != shape or out.get_device() != self._dev_index or not out.is_contiguous():
            raise ValueError(f"select_blocks: out must be a contiguous int32 {list(shape)} tensor on {self._dev}")
        batch = self._kv_batch("select_blocks", t, block_table, q_start, kv_len, max_q_len)
        a = SelectArgs(Batch(*batch), layer, dt, hq, n_blocks, first, last, qp, qts, qhs, self._bounds("select_blocks", bounds),
                       out.data_ptr(), 0, 0)
        n = self.L.kvt_select_scratch_bytes(self.h, C.byref(a))
        scratch = torch.empty(n, dtype=torch.uint8, device=self._dev) if n else None
        a.scratch, a.scratch_bytes = scratch.data_ptr() if n else None, n
        self._check(self.L.kvt_select_blocks(self.h, C.byref(a), self._kv_stream()), "select_blocks")
        return out

    def attend_blocks(self, layer, q, blocks, block_table, q_start, kv_len, scale=None, out=None, lse=None):
        """attend over the keys, up to each token's own, in the blocks that `blocks` (int32 [tokens, KV heads, n], contiguous, as
        select_blocks gives them) names for it. Entries below 0 and blocks behind the token's own count for nothing; lists may be in
        any order, without a block twice. Other arguments, precision and result as in attend."""
        done = self._attend_blocks_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                                          layer, q, blocks, block_table, q_start, kv_len, scale, out, lse)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "attend_blocks")
            return done
        # something is not as it should be (what, is said here), or only of another type than it might be
        torch = self.torch
        if layer < 0:
            raise ValueError("attend_blocks: layer cannot be negative")
        dt = self._kv_dtype(q, "attend_blocks")
        t, hq, d = q.shape if q.dim() == 3 else (0, 0, 0)
        qp, qts, qhs = self._kv_tensor(q, "attend_blocks: q", (t, hq, self.head_dim), q.dtype)
        if blocks.dtype is not torch.int32 or blocks.dim() != 3 or blocks.shape[:2] != (t, self.n_kv_heads) or \
                blocks.get_device() != self._dev_index or not blocks.is_contiguous():
            raise ValueError(f"attend_blocks: blocks must be a contiguous int32 [{t}, {self.n_kv_heads}, n] tensor on {self._dev}")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            op, ots, ohs = out.data_ptr(), hq * d, d
        else:
            op, ots, ohs = self._kv_tensor(out, "attend_blocks: out", (t, hq, d), q.dtype)
            if (ots == 0 and t > 1) or (ohs == 0 and hq > 1):
                raise ValueError("attend_blocks: out is a broadcast tensor")
        lsep = self._kv_lse("attend_blocks", lse, t, hq) if lse is not None else 0
        batch = self._kv_batch("attend_blocks", t, block_table, q_start, kv_len, 0)
        a = AttendBlocksArgs(Batch(*batch), layer, dt, hq, blocks.shape[2], self._kv_scale(scale), 0, qp, op, lsep, qts, qhs, ots, ohs,
                             blocks.data_ptr())
        self._check(self.L.kvt_attend_blocks(self.h, C.byref(a), self._kv_stream()), "attend_blocks")
        return out

    def weigh_blocks(self, layer, q, lse, block_table, q_start, kv_len, max_q_len=None, causal=True, window=None, scale=None,
                     weights=None, keep=1.0, out=None):
        """Attention weight per block, float32 [sequences, blocks of a table row]: keep * weights plus the sum, over the sequence's new
        tokens, query heads and the block's keys, of the weights exp(scale q k - lse) that attend gave them. q, lse, causal, window
        and scale are those of that call of attend; the lse of attend_blocks will not do, which is of the listed keys alone (blocks that
        were not listed would be weighed too heavily). weights: from earlier steps or layers (none: zeros); out: written if given, may be
        `weights`. Blocks behind kv_len get 0. max_q_len: most new tokens of one sequence, if known (chooses the kernel; results agree
        within their rounding). Asynchronous on the current stream. No backward pass, as in attend."""
        done = self._weigh_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                                  layer, q, lse, block_table, q_start, kv_len, max_q_len, causal, window, scale, weights, keep, out)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "weigh_blocks")
            return done
        # something is not as it should be (what, is said here), or only of another type than it might be
        torch = self.torch
        if layer < 0 or (max_q_len or 0) < 0 or (window or 0) < 0:
            raise ValueError("weigh_blocks: layer, max_q_len and window cannot be negative")
        dt = self._kv_dtype(q, "weigh_blocks")
        t, hq, d = q.shape if q.dim() == 3 else (0, 0, 0)
        qp, qts, qhs = self._kv_tensor(q, "weigh_blocks: q", (t, hq, self.head_dim), q.dtype)
        lsep = self._kv_lse("weigh_blocks", lse, t, hq)
        batch = self._kv_batch("weigh_blocks", t, block_table, q_start, kv_len, max_q_len)
        shape = tuple(block_table.shape)
        wp, ws = self._kv_rows("weigh_blocks: weights", weights, torch.float32, shape) if weights is not None else (0, 0)
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=self._dev)
        op, os_ = self._kv_rows("weigh_blocks: out", out, torch.float32, shape)
        if os_ < shape[1] and shape[0] > 1:
            raise ValueError("weigh_blocks: rows of out overlap")
        if wp == op and ws != os_ and shape[0] > 1:
            raise ValueError("weigh_blocks: out in the place of weights needs its strides")
        a = WeighArgs(Batch(*batch), layer, dt, hq, 0 if causal else ATTN_FULL, window or 0, self._kv_scale(scale), keep, 0, qp, lsep, qts,
                      qhs, wp, op, ws, os_, 0, 0)
        n = self.L.kvt_weigh_scratch_bytes(self.h, C.byref(a))
        scratch = torch.empty(n, dtype=torch.uint8, device=self._dev) if n else None
        a.scratch, a.scratch_bytes = scratch.data_ptr() if n else None, n
        self._check(self.L.kvt_weigh_blocks(self.h, C.byref(a), self._kv_stream()), "weigh_blocks")
        return out

    def evict_blocks(self, weights, block_table, kv_len, n_blocks, first=1, last=2, out=None):
        """Shortens the table rows of sequences that hold more than n_blocks blocks (a partly filled last one counts): the `first` first,
        the `last` last and the heaviest others stay, in order; of equal weights the lower numbers. Returns (block_table, kv_len,
        weights, evicted): rows of what stays, then -1 (weights: 0); lengths, 16 per block that left shorter; the slots that left,
        then -1. out: four tensors to write, of which the first three may be block_table, kv_len and weights themselves. Slots of the
        HBM tier go back with release(). Keys stay rotated by their old positions: append_kv needs `positions` from here on.
        Asynchronous on the current stream."""
        done = NotImplemented if out is not None else \
            self._evict_native(self.h and self.h.value, self._raw_stream(self._dev_index), self._dev_index, self.n_kv_heads, self.head_dim,
                               weights, block_table, kv_len, n_blocks, first, last)
        if done is not NotImplemented:
            if type(done) is int:
                self._check(done, "evict_blocks")
            return done
        # something is not as it should be (what, is said here), or only of another type than it might be
        torch = self.torch
        if min(n_blocks, first, last) < 0:
            raise ValueError("evict_blocks: n_blocks, first and last cannot be negative")
        if block_table.dim() != 2:
            raise ValueError("evict_blocks: block_table [sequences, blocks] expected")
        shape = tuple(block_table.shape)
        tp, ts = self._kv_rows("evict_blocks: block_table", block_table, torch.int32, shape)
        wp, ws = self._kv_rows("evict_blocks: weights", weights, torch.float32, shape)
        if out is None:
            out = (torch.empty(shape, dtype=torch.int32, device=self._dev), torch.empty(shape[0], dtype=torch.int32, device=self._dev),
                   torch.empty(shape, dtype=torch.float32, device=self._dev), torch.empty(shape, dtype=torch.int32, device=self._dev))
        table_out, len_out, w_out, evicted = out
        for x in (kv_len, len_out):
            if x.dtype is not torch.int32 or x.shape != shape[:1] or not x.is_contiguous() or x.get_device() != self._dev_index:
                raise ValueError(f"evict_blocks: lengths must be a contiguous int32 [{shape[0]}] tensor on {self._dev}")
        top, tos = self._kv_rows("evict_blocks: out block_table", table_out, torch.int32, shape)
        wop, wos = self._kv_rows("evict_blocks: out weights", w_out, torch.float32, shape)
        ep, es = self._kv_rows("evict_blocks: out evicted", evicted, torch.int32, shape)
        if shape[0] > 1 and min(tos, wos, es) < shape[1]:
            raise ValueError("evict_blocks: rows of an output overlap")
        if shape[0] > 1 and ((top == tp and tos != ts) or (wop == wp and wos != ws)):
            raise ValueError("evict_blocks: an output in the place of an input needs its strides")
        if evicted.numel() and ep in (tp, wp, top, wop):
            raise ValueError("evict_blocks: evicted needs a tensor of its own")
        a = EvictArgs(shape[0], shape[1], n_blocks, first, last, 0, tp, kv_len.data_ptr(), wp, ts, ws, top, len_out.data_ptr(), wop, ep, tos,
                      wos, es)
        self._check(self.L.kvt_evict_blocks(self.h, C.byref(a), self._kv_stream()), "evict_blocks")
        return table_out, len_out, w_out, evicted

    def kv_check(self):
        """Waits for the current stream and raises if one of the model-side calls met an id or a length outside its range. What a call
        that still runs on another stream meets is raised by this check or the next."""
        self._check(self.L.kvt_kv_check(self.h, self._kv_stream()), "kv_check")

    # ---- introspection --------------------------------------------------------------------------
    def get_stats(self):
        out = np.zeros(len(STATS_FIELDS), np.uint64)
        self._check(self.L.kvt_get_stats(self.h, _p(out)), "get_stats")
        return dict(zip(STATS_FIELDS, out.tolist()))

    def get_entries(self, tier):
        n = self._tier_size(tier)
        keys = np.zeros(n, np.uint64); stamp = np.zeros(n, np.uint32)
        depth = np.zeros(n, np.uint32); infl = np.zeros(n, np.uint32); link = np.zeros(n, np.uint32)
        self._check(self.L.kvt_get_entries(self.h, tier, _p(keys), _p(stamp), _p(depth), _p(infl), _p(link), n,
                                           _stream()), "get_entries")
        return {"key": keys, "stamp": stamp, "depth": depth, "inflight": infl, "link": link}

    def debug_load_resident_rc(self, keys, state, stamp, depth, slot, tier):
        k = np.ascontiguousarray(np.asarray(keys, np.uint64)); st = np.ascontiguousarray(np.asarray(state, np.uint8))
        sp, dp, sl = _u32(stamp), _u32(depth), _u32(slot)
        return self.L.kvt_debug_load_resident(self.h, _p(k), _p(st), _p(sp), _p(dp), _p(sl), tier, len(k), _stream())

    def debug_load_resident(self, *a):
        self._check(self.debug_load_resident_rc(*a), "debug_load_resident")

    # ---- payload access for the harness (producing KV is the model's job, not the engine's) -------
    def _chunks(self, tier, slot):
        if tier == TIER_HBM and self.pool_layout == LAYOUT_LAYER_MAJOR:
            return self.hbm_pool.view(self.n_chunks, self.n_hbm_blocks, self.chunk_bytes)[:, slot, :]
        pool = (self.hbm_pool, self.host_pool, self.remote_pool)[tier]
        return pool.view(-1, self.n_chunks, self.chunk_bytes)[slot]

    # Device-side counterpart of workloads.payload_pattern for large blocks (harness helpers, torch ops only).
    def _pattern(self, key):
        torch = self.torch
        if getattr(self, "_pat_base", None) is None:
            self._pat_base = (torch.arange(self.block_bytes // 4, dtype=torch.int64, device=self.device) * 0x9E3779B1) & 0xFFFFFFFF
        w = ((self._pat_base + (int(key) & 0xFFFFFFFF)) & 0xFFFFFFFF) ^ (int(key) >> 32)
        return w.to(torch.int32).view(torch.uint8).view(self.n_chunks, self.chunk_bytes)

    def fill_block_pattern(self, tier, slot, key):
        dst = self._chunks(tier, slot)
        dst.copy_(self._pattern(key).to(dst.device))

    def check_block_pattern(self, tier, slot, key) -> bool:
        self.torch.cuda.current_stream().synchronize()
        got = self._chunks(tier, slot).to(self.device)
        return bool(self.torch.equal(got, self._pattern(key)))

    def write_block(self, tier, slot, payload):
        t = self.torch.from_numpy(np.ascontiguousarray(np.asarray(payload, np.uint8))).view(self.n_chunks, self.chunk_bytes)
        dst = self._chunks(tier, slot)
        dst.copy_(t.to(dst.device))

    def read_block(self, tier, slot):
        self.torch.cuda.current_stream().synchronize()
        return self._chunks(tier, slot).contiguous().cpu().numpy().reshape(-1)
