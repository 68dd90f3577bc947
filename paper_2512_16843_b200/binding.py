"""ctypes binding of libllmcache.so: the same entry points as include/llmcache.h.

Only argument marshalling lives here.  Device memory and streams come from
PyTorch; every step of the probe runs in the library's CUDA kernels.  If the
shared library is missing or cannot be loaded the import of this module's
functions fails loudly -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# LLMCACHE_LIB selects another build of the same library (the range-checking debug build)
LIB_PATH = os.environ.get("LLMCACHE_LIB") or os.path.join(_HERE, "libllmcache.so")

OK = 0
ERR_ARG, ERR_SHAPE, ERR_NOMEM, ERR_CUDA, ERR_STATE, ERR_TIMEOUT, ERR_UNSUPPORTED, ERR_BOUNDS = -1, -2, -3, -4, -5, -6, -7, -8
F32, BF16 = 0, 1
GT, GE = 0, 1
LRU, LRU_STALENESS = 0, 1
EVICT_STALE, EVICT_IDLE, EVICT_ALL, EVICT_SLOTS = 0, 1, 2, 3
(WHAT_FP, WHAT_RB, WHAT_VALID, WHAT_LAST_USE, WHAT_INSERT_TICK, WHAT_HITS, WHAT_RATE,
 WHAT_RATE_EPOCH, WHAT_ACT, WHAT_TICK) = range(10)

EXPORTS = [
    "llmcache_abi_version", "llmcache_strerror", "llmcache_last_cuda_error", "llmcache_bank_bytes", "llmcache_bank_create",
    "llmcache_bank_destroy", "llmcache_fingerprint", "llmcache_probe", "llmcache_probe_fp",
    "llmcache_commit", "llmcache_evict", "llmcache_bank_export", "llmcache_bank_import",
    "llmcache_bank_stats", "llmcache_bank_status", "llmcache_bank_profile", "llmcache_bank_profile_read",
    "llmcache_fingerprint_static", "llmcache_fingerprint_static_error",
    "llmcache_layer_bytes", "llmcache_layer_create", "llmcache_layer_destroy", "llmcache_layer_forward",
    "llmcache_layer_status", "llmcache_infer", "llmcache_divergence_check", "llmcache_probe_simhash",
    "llmcache_pool", "llmcache_fingerprint_pooled", "llmcache_probe_pooled", "llmcache_bank_pool_out",
    "llmcache_infer_pooled", "llmcache_fingerprint_static_status", "llmcache_bank_debug_knobs",
    "llmcache_layer_debug_knobs", "llmcache_debug_bounds_build", "llmcache_bank_input_stable",
    "llmcache_shard_scan", "llmcache_shard_decide", "llmcache_embed",
    "llmcache_attention", "llmcache_attention_status", "llmcache_attention_debug_knobs", "llmcache_kv_bytes",
    "llmcache_kv_create", "llmcache_kv_destroy", "llmcache_kv_attention", "llmcache_kv_evict", "llmcache_kv_status",
    "llmcache_kv_debug_knobs", "llmcache_layer_score_mods", "llmcache_layer_extend",
]
KNOB_PRODUCER_IDLE = 1
FINGERPRINT_STATIC_MAX_FLOATS = 2 * 1024 * 1024
KERNEL_NAMES = ["pool", "project", "rownorm", "scan", "decide", "touch", "gather", "select", "scatter", "evict",
                "pool_finish"]


class BankDesc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("device", C.c_int32),
        ("capacity", C.c_uint32), ("seq_len", C.c_uint32), ("d_model", C.c_uint32), ("fp_dim", C.c_uint32),
        ("hidden_dtype", C.c_uint32), ("act_rows", C.c_uint32), ("max_batch", C.c_uint32),
        ("tau", C.c_float), ("cmp", C.c_uint32), ("policy", C.c_uint32),
        ("half_life_ticks", C.c_uint32), ("stale_floor_q8", C.c_uint32),
        ("min_age_ticks", C.c_uint32), ("max_idle_ticks", C.c_uint32), ("store_act", C.c_uint32),
        ("fused_pool", C.c_uint32),
        ("proj", C.c_void_p), ("center", C.c_void_p), ("arena", C.c_void_p), ("arena_bytes", C.c_size_t),
    ]


class ProbeIO(C.Structure):
    _fields_ = [
        ("hit", C.c_void_p), ("slot", C.c_void_p), ("score", C.c_void_p), ("hit_idx", C.c_void_p),
        ("miss_idx", C.c_void_p), ("counts", C.c_void_p), ("counts_host", C.c_void_p),
        ("fp", C.c_void_p), ("rq", C.c_void_p), ("h_miss", C.c_void_p), ("generation", C.c_uint64),
    ]


class LayerDesc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("device", C.c_int32), ("d_model", C.c_uint32), ("heads", C.c_uint32),
        ("ffn", C.c_uint32), ("seq_len", C.c_uint32), ("max_seqs", C.c_uint32), ("pre_ln", C.c_uint32),
        ("causal", C.c_uint32), ("tanh_gelu", C.c_uint32), ("eps", C.c_float),
        ("w_qkv", C.c_void_p), ("b_qkv", C.c_void_p), ("w_o", C.c_void_p), ("b_o", C.c_void_p),
        ("ln1_g", C.c_void_p), ("ln1_b", C.c_void_p), ("w_1", C.c_void_p), ("b_1", C.c_void_p),
        ("w_2", C.c_void_p), ("b_2", C.c_void_p), ("ln2_g", C.c_void_p), ("ln2_b", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class ScoreMods(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("causal", C.c_uint32), ("scale", C.c_float), ("cap", C.c_float),
        ("reach", C.c_uint32), ("mask_seqs", C.c_uint32), ("slopes", C.c_void_p), ("table", C.c_void_p), ("doc", C.c_void_p), ("prefix", C.c_void_p),
    ]


class Rows(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("seq_stride", C.c_int64), ("tok_stride", C.c_int64), ("head_stride", C.c_int64)]


class KVDesc(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("device", C.c_int32), ("heads", C.c_uint32), ("kv_heads", C.c_uint32),
        ("num_pages", C.c_uint32), ("page_size", C.c_uint32), ("max_seqs", C.c_uint32), ("max_rows", C.c_uint32),
        ("max_len", C.c_uint32), ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("page_stride", C.c_uint64),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t),
    ]


class KVChunk(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("n_seqs", C.c_uint32), ("n_rows", C.c_uint32), ("longest", C.c_uint32),
        ("cu_rows", C.c_void_p), ("lens", C.c_void_p), ("pages", C.c_void_p), ("pages_ld", C.c_uint32),
        ("decay", C.c_float), ("q", Rows), ("out", Rows), ("k_new", Rows), ("v_new", Rows), ("lse", C.c_void_p),
        ("weights", C.c_void_p), ("positions", C.c_void_p), ("first", C.c_void_p), ("side_ld", C.c_uint64),
        ("mods", C.POINTER(ScoreMods)),
    ]


class KVEviction(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("n_seqs", C.c_uint32), ("budget", C.c_uint32), ("recent", C.c_uint32),
        ("sinks", C.c_uint32), ("pages_ld", C.c_uint32), ("new_pages_ld", C.c_uint32), ("lens", C.c_void_p),
        ("pages", C.c_void_p), ("new_pages", C.c_void_p), ("new_lens", C.c_void_p), ("weights", C.c_void_p),
        ("positions", C.c_void_p), ("side_ld", C.c_uint64), ("new_weights", C.c_void_p), ("new_positions", C.c_void_p),
        ("new_side_ld", C.c_uint64), ("kept", C.c_void_p),
    ]


WEIGHT_NAMES = ("w_qkv", "b_qkv", "w_o", "b_o", "ln1_g", "ln1_b", "w_1", "b_1", "w_2", "b_2", "ln2_g", "ln2_b")


class Stats(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("probes", "sequences", "hits", "misses", "degenerate",
                                          "inserts", "evictions", "dropped", "flushed", "resident",
                                          "kernel_launches")]


class LLMCacheError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = lib().llmcache_last_cuda_error().decode() if status == ERR_CUDA else ""
        super().__init__(f"{where}: {strerror(status)} ({status}) {detail}")


_lib = None


def lib():
    """The loaded shared library (loads it on first use)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_16843_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, u32, i32p = C.c_void_p, C.c_uint32, C.c_void_p
        L.llmcache_abi_version.restype = C.c_uint32
        L.llmcache_abi_version.argtypes = []
        L.llmcache_strerror.restype = C.c_char_p
        L.llmcache_strerror.argtypes = [C.c_int]
        L.llmcache_last_cuda_error.restype = C.c_char_p
        L.llmcache_last_cuda_error.argtypes = []
        L.llmcache_embed.argtypes = [vp, C.c_uint64, u32, u32, C.c_int64, vp, vp, C.c_int32, vp, vp, C.c_float, vp, vp, vp]
        L.llmcache_bank_bytes.argtypes = [C.POINTER(BankDesc), C.POINTER(C.c_size_t)]
        L.llmcache_bank_create.argtypes = [C.POINTER(BankDesc), C.POINTER(vp)]
        L.llmcache_bank_destroy.argtypes = [vp]
        L.llmcache_fingerprint.argtypes = [vp, vp, u32, vp, vp, vp]
        L.llmcache_probe.argtypes = [vp, vp, u32, C.c_float, vp, C.POINTER(ProbeIO), vp]
        L.llmcache_probe_fp.argtypes = [vp, vp, u32, C.c_float, vp, C.POINTER(ProbeIO), vp]
        L.llmcache_probe_simhash.argtypes = [vp, vp, u32, C.c_float, vp, C.POINTER(ProbeIO), vp]
        L.llmcache_commit.argtypes = [vp, vp, C.POINTER(ProbeIO), vp, i32p, vp]
        L.llmcache_evict.argtypes = [vp, u32, vp, u32, vp, vp]
        L.llmcache_bank_export.argtypes = [vp, u32, vp, C.c_size_t, vp]
        L.llmcache_bank_import.argtypes = [vp, u32, vp, C.c_size_t, vp]
        L.llmcache_bank_stats.argtypes = [vp, C.POINTER(Stats)]
        L.llmcache_bank_status.argtypes = [vp]
        L.llmcache_bank_profile.argtypes = [vp, C.c_int]
        L.llmcache_bank_profile_read.argtypes = [vp, u32, C.POINTER(C.c_double), C.POINTER(C.c_uint64)]
        L.llmcache_layer_bytes.argtypes = [C.POINTER(LayerDesc), C.POINTER(C.c_size_t)]
        L.llmcache_layer_create.argtypes = [C.POINTER(LayerDesc), C.POINTER(vp)]
        L.llmcache_layer_destroy.argtypes = [vp]
        L.llmcache_layer_forward.argtypes = [vp, vp, u32, vp, vp, vp]
        L.llmcache_layer_status.argtypes = [vp]
        L.llmcache_infer.argtypes = [C.POINTER(vp), C.POINTER(vp), u32, vp, u32, C.c_float, vp, vp, vp, vp,
                                     C.POINTER(ProbeIO), C.POINTER(vp), vp]
        L.llmcache_divergence_check.argtypes = [vp, vp, vp, C.POINTER(ProbeIO), u32, C.c_float, vp, vp, vp, vp, vp]
        L.llmcache_pool.argtypes = [vp, vp, u32, vp, u32, vp]
        L.llmcache_fingerprint_pooled.argtypes = [vp, vp, u32, u32, vp, vp, vp]
        L.llmcache_probe_pooled.argtypes = [vp, vp, u32, vp, u32, C.c_float, vp, C.POINTER(ProbeIO), vp]
        L.llmcache_bank_pool_out.argtypes = [vp, vp, u32]
        L.llmcache_infer_pooled.argtypes = [C.POINTER(vp), C.POINTER(vp), u32, vp, u32, C.c_float, vp, vp, vp, vp,
                                            C.POINTER(ProbeIO), vp, C.POINTER(vp), vp]
        L.llmcache_fingerprint_static.argtypes = [vp, u32, u32, u32, u32, u32, vp, vp, vp, vp, vp]
        L.llmcache_fingerprint_static_error.restype = C.c_char_p
        L.llmcache_fingerprint_static_error.argtypes = []
        L.llmcache_fingerprint_static_status.argtypes = []
        L.llmcache_debug_bounds_build.argtypes = []
        L.llmcache_bank_input_stable.argtypes = [vp, C.c_int]
        L.llmcache_shard_scan.argtypes = [vp, vp, u32, u32, vp, vp]
        L.llmcache_shard_decide.argtypes = [vp, vp, u32, C.c_float, u32, u32, vp, C.POINTER(ProbeIO), vp]
        L.llmcache_bank_debug_knobs.argtypes = [vp, C.c_uint64, u32]
        L.llmcache_layer_debug_knobs.argtypes = [vp, C.c_uint64, u32]
        # (structs of the calls that a step makes are packed into bytes: a fifth of the time of a ctypes structure)
        L.llmcache_attention.argtypes = [vp, vp, vp, vp, u32, u32, u32, u32, vp, vp, vp, vp]
        L.llmcache_attention_status.argtypes = []
        L.llmcache_attention_debug_knobs.argtypes = [C.c_uint64, u32]
        L.llmcache_kv_bytes.argtypes = [C.POINTER(KVDesc), C.POINTER(C.c_size_t)]
        L.llmcache_kv_create.argtypes = [C.POINTER(KVDesc), C.POINTER(vp)]
        L.llmcache_kv_destroy.argtypes = [vp]
        L.llmcache_kv_attention.argtypes = [vp, vp, vp]
        L.llmcache_kv_evict.argtypes = [vp, vp, vp]
        L.llmcache_kv_status.argtypes = [vp]
        L.llmcache_kv_debug_knobs.argtypes = [vp, C.c_uint64, u32]
        L.llmcache_layer_score_mods.argtypes = [vp, C.POINTER(ScoreMods)]
        L.llmcache_layer_extend.argtypes = [vp, vp, vp, C.POINTER(KVChunk), vp, vp]
        for name in EXPORTS:
            if name not in ("llmcache_abi_version", "llmcache_strerror", "llmcache_last_cuda_error",
                            "llmcache_fingerprint_static_error"):
                getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def strerror(status: int) -> str:
    return lib().llmcache_strerror(int(status)).decode()


def _check(rc: int, where: str):
    if rc != OK:
        raise LLMCacheError(rc, where)


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# the current stream's handle without a Stream object around it (a tenth of the time), where torch has that
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, device=None) -> Optional[int]:
    """Handle of a stream; None: the current one of the current (or the given) device."""
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device() if device is None else device)
        return torch.cuda.current_stream(device).cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ----------------------------------------------------------------------------
# Entry points, named as in llmcache.h
# ----------------------------------------------------------------------------
def llmcache_abi_version() -> int:
    return int(lib().llmcache_abi_version())


def make_desc(*, device=0, capacity, seq_len, d_model, fp_dim, hidden_dtype=BF16, act_rows=0, max_batch,
              tau=0.9, cmp=GT, policy=LRU_STALENESS, half_life_ticks=0, stale_floor_q8=0, min_age_ticks=0,
              max_idle_ticks=0, store_act=1, fused_pool=0, proj=None, center=None, arena=None, arena_bytes=0) -> BankDesc:
    d = BankDesc()
    d.struct_size = C.sizeof(BankDesc)
    d.device, d.capacity, d.seq_len, d.d_model, d.fp_dim = device, capacity, seq_len, d_model, fp_dim
    d.hidden_dtype, d.act_rows, d.max_batch = hidden_dtype, act_rows, max_batch
    d.tau, d.cmp, d.policy = tau, cmp, policy
    d.half_life_ticks, d.stale_floor_q8 = half_life_ticks, stale_floor_q8
    d.min_age_ticks, d.max_idle_ticks, d.store_act = min_age_ticks, max_idle_ticks, store_act
    d.fused_pool = fused_pool
    d.proj, d.center, d.arena, d.arena_bytes = _ptr(proj), _ptr(center), _ptr(arena), arena_bytes
    return d


def llmcache_bank_bytes(desc: BankDesc) -> int:
    out = C.c_size_t(0)
    _check(lib().llmcache_bank_bytes(C.byref(desc), C.byref(out)), "llmcache_bank_bytes")
    return int(out.value)


def llmcache_bank_create(desc: BankDesc) -> int:
    out = C.c_void_p(None)
    _check(lib().llmcache_bank_create(C.byref(desc), C.byref(out)), "llmcache_bank_create")
    return out.value


def llmcache_bank_destroy(bank: int) -> None:
    _check(lib().llmcache_bank_destroy(bank), "llmcache_bank_destroy")


def llmcache_fingerprint(bank, h_in, B, fp, rq, stream=None) -> None:
    _check(lib().llmcache_fingerprint(bank, _ptr(h_in), B, _ptr(fp), _ptr(rq), _stream(stream)),
           "llmcache_fingerprint")


def llmcache_fingerprint_static(h_in, hidden_dtype, B, seq_len, d_model, fp_dim, proj, center, fp, rq,
                                stream=None) -> None:
    """Fingerprint on the current device without a bank and without any allocation by the library
    (for callers whose device memory is all spoken for).  Raises LLMCacheError with the library's
    explanation when the call is refused, e.g. because the batch exceeds the fixed scratch."""
    rc = lib().llmcache_fingerprint_static(_ptr(h_in), hidden_dtype, B, seq_len, d_model, fp_dim, _ptr(proj),
                                           _ptr(center), _ptr(fp), _ptr(rq), _stream(stream))
    if rc != OK:
        err = LLMCacheError(rc, "llmcache_fingerprint_static")
        err.args = (err.args[0] + " " + lib().llmcache_fingerprint_static_error().decode(),)
        raise err


def llmcache_probe(bank, h_in, B, tau, h_out, io: ProbeIO, stream=None) -> None:
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_probe(bank, _ptr(h_in), B, tau, _ptr(h_out), C.byref(io), _stream(stream)),
           "llmcache_probe")


def llmcache_probe_simhash(bank, h_in, B, tau, h_out, io: ProbeIO, stream=None) -> None:
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_probe_simhash(bank, _ptr(h_in), B, tau, _ptr(h_out), C.byref(io), _stream(stream)),
           "llmcache_probe_simhash")


def llmcache_probe_fp(bank, h_in, B, tau, h_out, io: ProbeIO, stream=None) -> None:
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_probe_fp(bank, _ptr(h_in), B, tau, _ptr(h_out), C.byref(io), _stream(stream)),
           "llmcache_probe_fp")


def llmcache_pool(bank, h_in, B, pooled, ld, stream=None) -> None:
    _check(lib().llmcache_pool(bank, _ptr(h_in), B, _ptr(pooled), ld, _stream(stream)), "llmcache_pool")


def llmcache_fingerprint_pooled(bank, pooled, ld, B, fp, rq, stream=None) -> None:
    _check(lib().llmcache_fingerprint_pooled(bank, _ptr(pooled), ld, B, _ptr(fp), _ptr(rq), _stream(stream)),
           "llmcache_fingerprint_pooled")


def llmcache_probe_pooled(bank, pooled, ld, h_in, B, tau, h_out, io: ProbeIO, stream=None) -> None:
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_probe_pooled(bank, _ptr(pooled), ld, _ptr(h_in), B, tau, _ptr(h_out), C.byref(io),
                                       _stream(stream)), "llmcache_probe_pooled")


def llmcache_bank_pool_out(bank, pooled_out, ld) -> None:
    _check(lib().llmcache_bank_pool_out(bank, _ptr(pooled_out), ld), "llmcache_bank_pool_out")


def llmcache_commit(bank, miss_out, io: ProbeIO, h_out, new_slot, stream=None) -> None:
    _check(lib().llmcache_commit(bank, _ptr(miss_out), C.byref(io), _ptr(h_out), _ptr(new_slot), _stream(stream)),
           "llmcache_commit")


def llmcache_evict(bank, mode, slots=None, n=0, n_evicted_dev=None, stream=None) -> None:
    _check(lib().llmcache_evict(bank, mode, _ptr(slots), n, _ptr(n_evicted_dev), _stream(stream)), "llmcache_evict")


def llmcache_bank_export(bank, what, ptr, nbytes, stream=None) -> None:
    _check(lib().llmcache_bank_export(bank, what, _ptr(ptr), nbytes, _stream(stream)), "llmcache_bank_export")


def llmcache_bank_import(bank, what, ptr, nbytes, stream=None) -> None:
    _check(lib().llmcache_bank_import(bank, what, _ptr(ptr), nbytes, _stream(stream)), "llmcache_bank_import")


def llmcache_bank_stats(bank) -> dict:
    s = Stats()
    _check(lib().llmcache_bank_stats(bank, C.byref(s)), "llmcache_bank_stats")
    return {n: int(getattr(s, n)) for n, _ in Stats._fields_}


def llmcache_bank_status(bank) -> int:
    return int(lib().llmcache_bank_status(bank))


def llmcache_bank_debug_knobs(bank, wait_limit_ns: int, flags: int) -> None:
    _check(lib().llmcache_bank_debug_knobs(bank, wait_limit_ns, flags), "llmcache_bank_debug_knobs")


def llmcache_layer_debug_knobs(layer, wait_limit_ns: int, flags: int) -> None:
    _check(lib().llmcache_layer_debug_knobs(layer, wait_limit_ns, flags), "llmcache_layer_debug_knobs")


def llmcache_debug_bounds_build() -> bool:
    return bool(lib().llmcache_debug_bounds_build())


def llmcache_fingerprint_static_status() -> int:
    return int(lib().llmcache_fingerprint_static_status())


def llmcache_shard_scan(bank, fp, B, slot_base, words, stream=None) -> None:
    _check(lib().llmcache_shard_scan(bank, _ptr(fp), B, slot_base, _ptr(words), _stream(stream)), "llmcache_shard_scan")


def llmcache_shard_decide(bank, words, B, tau, slot_base, n_total, h_out, io: ProbeIO, stream=None) -> None:
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_shard_decide(bank, _ptr(words), B, tau, slot_base, n_total, _ptr(h_out), C.byref(io),
                                       _stream(stream)), "llmcache_shard_decide")


def llmcache_bank_profile(bank, enable: bool) -> None:
    _check(lib().llmcache_bank_profile(bank, 1 if enable else 0), "llmcache_bank_profile")


def llmcache_bank_profile_read(bank, kernel_id: int):
    ms, n = C.c_double(0.0), C.c_uint64(0)
    _check(lib().llmcache_bank_profile_read(bank, kernel_id, C.byref(ms), C.byref(n)), "llmcache_bank_profile_read")
    return float(ms.value), int(n.value)


# ----------------------------------------------------------------------------
# Buffer holders (allocation and marshalling only)
# ----------------------------------------------------------------------------
class ProbeBuffers:
    """Device buffers for one probe of up to B sequences, plus the C struct that points at them."""

    def __init__(self, B: int, fp_dim: int, device="cuda", pinned_counts: bool = True,
                 h_miss: Optional[torch.Tensor] = None):
        dev = torch.device(device)
        Bm = max(B, 1)
        self.B = B
        self.hit = torch.zeros(Bm, dtype=torch.uint8, device=dev)
        self.slot = torch.full((Bm,), -1, dtype=torch.int32, device=dev)
        self.score = torch.zeros(Bm, dtype=torch.float32, device=dev)
        self.hit_idx = torch.zeros(Bm, dtype=torch.int32, device=dev)
        self.miss_idx = torch.zeros(Bm, dtype=torch.int32, device=dev)
        self.counts = torch.zeros(2, dtype=torch.int32, device=dev)
        self.counts_host = torch.zeros(2, dtype=torch.int32).pin_memory() if pinned_counts else None
        self.fp = torch.zeros((Bm, fp_dim), dtype=torch.bfloat16, device=dev)
        self.rq = torch.zeros(Bm, dtype=torch.float32, device=dev)
        self.new_slot = torch.full((Bm,), -1, dtype=torch.int32, device=dev)
        self.h_miss = h_miss
        self.io = ProbeIO()
        self.io.hit, self.io.slot, self.io.score = self.hit.data_ptr(), self.slot.data_ptr(), self.score.data_ptr()
        self.io.hit_idx, self.io.miss_idx = self.hit_idx.data_ptr(), self.miss_idx.data_ptr()
        self.io.counts = self.counts.data_ptr()
        self.io.counts_host = self.counts_host.data_ptr() if pinned_counts else None
        self.io.fp, self.io.rq = self.fp.data_ptr(), self.rq.data_ptr()
        self.io.h_miss = h_miss.data_ptr() if h_miss is not None else None
        self.io.generation = 0


_WHAT_DTYPE = {
    WHAT_FP: torch.bfloat16, WHAT_RB: torch.float32, WHAT_VALID: torch.uint8, WHAT_LAST_USE: torch.int32,
    WHAT_INSERT_TICK: torch.int32, WHAT_HITS: torch.int32, WHAT_RATE: torch.int32, WHAT_RATE_EPOCH: torch.int32,
    WHAT_ACT: torch.bfloat16,
}


class Bank:
    """Owner of one llmcache_bank_t handle (one transformer layer's cache)."""

    def __init__(self, **kw):
        self._proj = kw.get("proj")
        self._center = kw.get("center")
        self.desc = make_desc(**kw)
        self.handle = llmcache_bank_create(self.desc)
        self.N, self.n, self.d, self.k = self.desc.capacity, self.desc.seq_len, self.desc.d_model, self.desc.fp_dim
        self.act_rows = self.desc.act_rows or self.desc.capacity
        self.device = torch.device("cuda", self.desc.device)

    def close(self):
        if getattr(self, "handle", None):
            llmcache_bank_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _shape(self, what):
        if what == WHAT_FP:
            return (self.N, self.k)
        if what == WHAT_ACT:
            return (self.act_rows, self.n * self.d)
        return (self.N,)

    def export(self, what) -> torch.Tensor:
        """Copy of one bank array as a host tensor (synchronises)."""
        if what == WHAT_TICK:
            t = torch.zeros(1, dtype=torch.int64)
            llmcache_bank_export(self.handle, what, t.data_ptr(), 8)
            return t
        dev = torch.empty(self._shape(what), dtype=_WHAT_DTYPE[what], device=self.device)
        llmcache_bank_export(self.handle, what, dev.data_ptr(), dev.numel() * dev.element_size())
        torch.cuda.synchronize(self.device)
        return dev.cpu()

    def import_(self, what, t: torch.Tensor):
        if what == WHAT_TICK:
            t = t.to(torch.int64).contiguous()
            llmcache_bank_import(self.handle, what, t.data_ptr(), 8)
            return
        t = t.to(device=self.device).contiguous()
        llmcache_bank_import(self.handle, what, t.data_ptr(), t.numel() * t.element_size())
        torch.cuda.synchronize(self.device)

    def probe(self, h_in, bufs: ProbeBuffers, h_out=None, tau=None, B=None, stream=None):
        B = h_in.shape[0] if B is None else B
        llmcache_probe(self.handle, h_in, B, tau, h_out, bufs.io, stream)

    def probe_pooled(self, pooled, bufs: ProbeBuffers, B, h_out=None, tau=None, h_in=None, stream=None):
        llmcache_probe_pooled(self.handle, pooled, pooled.stride(0), h_in, B, tau, h_out, bufs.io, stream)

    def pool_out(self, pooled_out):
        """Position means of the rows written by the next probes + commits go to pooled_out [B, >=d] f32
        (None switches it off)."""
        llmcache_bank_pool_out(self.handle, pooled_out, 0 if pooled_out is None else pooled_out.stride(0))
        self._pool_out = pooled_out

    def pool(self, h_in, pooled, B=None, stream=None):
        llmcache_pool(self.handle, h_in, h_in.shape[0] if B is None else B, pooled, pooled.stride(0), stream)

    def fingerprint_pooled(self, pooled, fp, rq, B=None, stream=None):
        llmcache_fingerprint_pooled(self.handle, pooled, pooled.stride(0), pooled.shape[0] if B is None else B,
                                    fp, rq, stream)

    def probe_fp(self, bufs: ProbeBuffers, B, h_out=None, tau=None, h_in=None, stream=None):
        llmcache_probe_fp(self.handle, h_in, B, tau, h_out, bufs.io, stream)

    def commit(self, miss_out, bufs: ProbeBuffers, h_out=None, stream=None):
        llmcache_commit(self.handle, miss_out, bufs.io, h_out, bufs.new_slot, stream)

    def evict(self, mode, slots: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None, stream=None):
        n = 0 if slots is None else slots.numel()
        llmcache_evict(self.handle, mode, slots, n, count, stream)

    def stats(self) -> dict:
        return llmcache_bank_stats(self.handle)

    def status(self) -> int:
        return llmcache_bank_status(self.handle)

    def debug_knobs(self, wait_limit_ns: int = 0, flags: int = 0):
        llmcache_bank_debug_knobs(self.handle, wait_limit_ns, flags)

    def input_stable(self, stable: bool = True):
        """Promise that probe inputs are never written by the kernel preceding the probe in its stream."""
        _check(lib().llmcache_bank_input_stable(self.handle, 1 if stable else 0), "llmcache_bank_input_stable")

    def profile(self, enable: bool):
        llmcache_bank_profile(self.handle, enable)

    def profile_read(self) -> dict:
        """{kernel name: (total ms, launches)} since the last read."""
        return {name: llmcache_bank_profile_read(self.handle, i) for i, name in enumerate(KERNEL_NAMES)}


# ----------------------------------------------------------------------------
# Miss-path transformer layer and the layer-wise caching loop
# ----------------------------------------------------------------------------
def llmcache_layer_bytes(desc: LayerDesc) -> int:
    out = C.c_size_t(0)
    _check(lib().llmcache_layer_bytes(C.byref(desc), C.byref(out)), "llmcache_layer_bytes")
    return int(out.value)


def llmcache_layer_create(desc: LayerDesc) -> int:
    out = C.c_void_p(None)
    _check(lib().llmcache_layer_create(C.byref(desc), C.byref(out)), "llmcache_layer_create")
    return out.value


def llmcache_layer_destroy(layer: int) -> None:
    _check(lib().llmcache_layer_destroy(layer), "llmcache_layer_destroy")


def llmcache_layer_forward(layer, x, n_seqs, n_seqs_dev, out, stream=None) -> None:
    _check(lib().llmcache_layer_forward(layer, _ptr(x), n_seqs, _ptr(n_seqs_dev), _ptr(out), _stream(stream)),
           "llmcache_layer_forward")


def llmcache_layer_status(layer) -> int:
    return int(lib().llmcache_layer_status(layer))


def llmcache_embed(tokens, tok_emb, pos_emb, h0, *, layer_norm=True, ln_gain=None, ln_bias=None, eps=1e-5,
                   bad_ids=None, stream=None) -> None:
    """h0 = E(X) of Algorithm 1: token + position embeddings, optionally layer-normed.  tokens: int64 [S, n] on the
    device; tok_emb bf16 [vocab, d]; pos_emb bf16 [n, d] or None; h0 bf16 [S, n, d]."""
    S, n = tokens.shape
    vocab, d = tok_emb.shape
    _check(lib().llmcache_embed(_ptr(tokens), S, n, d, vocab, _ptr(tok_emb), _ptr(pos_emb), int(layer_norm),
                                _ptr(ln_gain), _ptr(ln_bias), eps, _ptr(h0), _ptr(bad_ids), _stream(stream)),
           "llmcache_embed")


def llmcache_infer(banks, layers, h0, B, tau, buf_a, buf_b, h_miss, miss_out, io, stream=None) -> int:
    """Algorithm 1 over all layers; returns the device address (buf_a or buf_b) that will hold h_L."""
    n = len(layers)
    larr = (C.c_void_p * n)(*layers)
    barr = (C.c_void_p * n)(*banks) if banks is not None else None
    final = C.c_void_p(None)
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_infer(barr, larr, n, _ptr(h0), B, tau, _ptr(buf_a), _ptr(buf_b), _ptr(h_miss),
                                _ptr(miss_out), C.byref(io) if io is not None else None, C.byref(final),
                                _stream(stream)), "llmcache_infer")
    return final.value


def llmcache_infer_pooled(banks, layers, h0, B, tau, buf_a, buf_b, h_miss, miss_out, io, pooled, stream=None) -> int:
    """Algorithm 1 with fingerprint-on-write; returns the device address that will hold h_L."""
    n = len(layers)
    larr = (C.c_void_p * n)(*layers)
    barr = (C.c_void_p * n)(*banks)
    final = C.c_void_p(None)
    tau = float("nan") if tau is None else tau
    _check(lib().llmcache_infer_pooled(barr, larr, n, _ptr(h0), B, tau, _ptr(buf_a), _ptr(buf_b), _ptr(h_miss),
                                       _ptr(miss_out), C.byref(io), _ptr(pooled), C.byref(final), _stream(stream)),
           "llmcache_infer_pooled")
    return final.value


def llmcache_divergence_check(bank, layer, h_in, io, stride, bound, h_sample, out_sample, rel_out, counters_dev,
                              stream=None) -> None:
    _check(lib().llmcache_divergence_check(bank, layer, _ptr(h_in), C.byref(io), stride, bound, _ptr(h_sample),
                                           _ptr(out_sample), _ptr(rel_out), _ptr(counters_dev), _stream(stream)),
           "llmcache_divergence_check")


class Layer:
    """Owner of one llmcache_layer_t handle; keeps the weight tensors alive (the library borrows them)."""

    def __init__(self, weights: dict, *, device=0, heads, seq_len, max_seqs, pre_ln=False, causal=False,
                 tanh_gelu=False, eps=1e-5, workspace: Optional[torch.Tensor] = None):
        self.weights = {k: weights[k].contiguous() for k in WEIGHT_NAMES}
        d = LayerDesc()
        d.struct_size = C.sizeof(LayerDesc)
        d.device = device
        d.d_model = self.weights["w_o"].shape[0]
        d.heads, d.ffn, d.seq_len, d.max_seqs = heads, self.weights["w_1"].shape[0], seq_len, max_seqs
        d.pre_ln, d.causal, d.tanh_gelu, d.eps = int(pre_ln), int(causal), int(tanh_gelu), eps
        for k in WEIGHT_NAMES:
            setattr(d, k, self.weights[k].data_ptr())
        self.workspace = workspace
        if workspace is not None:
            d.workspace, d.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        self.desc = d
        self.handle = llmcache_layer_create(d)

    def forward(self, x, out, n_seqs=None, n_seqs_dev=None, stream=None):
        llmcache_layer_forward(self.handle, x, x.shape[0] if n_seqs is None else n_seqs, n_seqs_dev, out, stream)

    def score_mods(self, mods: Optional[ScoreMods]):
        """Score modifiers (make_score_mods) of the forward and extend calls that follow; None switches them off.  doc is
        [n_seqs, seq_len of the layer], and forward calls bring at most that many sequences."""
        if mods is not None:
            _check_mods(mods, self.desc.heads, self.desc.device, layer_len=self.desc.seq_len)
        llmcache_layer_score_mods(self.handle, mods)
        self._mods = mods                                # keeps the arrays alive

    def extend(self, cache: "KVCache", x, out, *, cu_rows, lens, pages, longest=0, weights=None, decay=1.0, positions=None,
               first=None, stream=None):
        """The layer on new tokens: x, out [n_rows, d]; the other arguments as in KVCache.attention (rows beyond `longest` get
        the layer's result for an attention of zero)."""
        chunk = cache.chunk(x.shape[0], cu_rows=cu_rows, lens=lens, pages=pages, longest=longest, weights=weights, decay=decay,
                            positions=positions, first=first)
        _want(x, torch.bfloat16, 2, "x")
        _want(out, torch.bfloat16, 2, "out")
        if not (x.is_contiguous() and out.is_contiguous() and x.shape == out.shape and x.shape[1] == self.desc.d_model):
            raise LLMCacheError(ERR_SHAPE, "llmcache_layer_extend: x and out are dense [n_rows, d_model]")
        _same_device(cache.device, x, out)
        _check(lib().llmcache_layer_extend(self.handle, cache.handle, _ptr(x), C.byref(chunk), _ptr(out), _stream(stream, cache.device)),
               "llmcache_layer_extend")

    def status(self) -> int:
        return llmcache_layer_status(self.handle)

    def debug_knobs(self, wait_limit_ns: int = 0, flags: int = 0):
        llmcache_layer_debug_knobs(self.handle, wait_limit_ns, flags)

    def close(self):
        if getattr(self, "handle", None):
            llmcache_layer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ----------------------------------------------------------------------------
# Attention with score modifiers, paged key/value cache, eviction
# ----------------------------------------------------------------------------
def _want(t, dtype, dim, name):
    """Type and rank of a tensor argument; strides that the C side cannot see."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != dim:
        raise LLMCacheError(ERR_ARG, f"{name}: a {dtype} tensor of {dim} dimensions is expected")


def _dense(t, dtype, dim, name, optional=False):
    if t is None and optional:
        return
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != dim or not t.is_contiguous():
        raise LLMCacheError(ERR_ARG, f"{name}: a contiguous {dtype} tensor of {dim} dimensions is expected")


_BF16 = torch.bfloat16


def _other_device(t, device):
    raise LLMCacheError(ERR_ARG, f"a tensor on device {t.get_device()} where device {device} is expected (-1: the host)")


def _rows(t, name, dim, shape, device):
    """[seq, token, head, 64] or [token, head, 64] view of any strides: (address, strides of sequence, token and head)."""
    if not isinstance(t, torch.Tensor) or t.dtype is not _BF16 or t.dim() != dim:
        raise LLMCacheError(ERR_ARG, f"{name}: a {_BF16} tensor of {dim} dimensions is expected")
    st, sh = t.stride(), t.shape
    if sh[-1] != 64 or (st[-1] != 1 and t.numel()):
        raise LLMCacheError(ERR_SHAPE, f"{name}: the last dimension holds 64 neighbouring elements")
    if shape is not None and sh != shape:
        raise LLMCacheError(ERR_SHAPE, f"{name}: {tuple(sh)} where {tuple(shape)} is expected")
    if t.get_device() != device:
        _other_device(t, device)
    return (t.data_ptr(), *st[:3]) if dim == 4 else (t.data_ptr(), 0, st[0], st[1])


def _addr(t, dtype, shape, name, device) -> int:
    """Address of a dense tensor of one type, shape and device; None: 0.  (A length of -1 may be anything.)"""
    if t is None:
        return 0
    try:
        if t.dtype is dtype and t.get_device() == device and t.is_contiguous():
            have = t.shape
            if have == shape:
                return t.data_ptr()
            if shape[-1] < 0 and len(have) == len(shape) and have[:-1] == shape[:-1]:
                return t.data_ptr()
    except AttributeError:
        pass
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != len(shape) or not t.is_contiguous():
        raise LLMCacheError(ERR_ARG, f"{name}: a contiguous {dtype} tensor of {len(shape)} dimensions is expected")
    if t.get_device() != device:
        _other_device(t, device)
    raise LLMCacheError(ERR_SHAPE, f"{name}: {tuple(t.shape)} where {shape} is expected")


class _Packed(struct.Struct):
    """A C structure as bytes; numbers that do not fit their fields are refused."""

    def __call__(self, *values) -> bytes:
        try:
            return self.pack(*values)
        except struct.error as e:
            raise LLMCacheError(ERR_ARG, str(e)) from None


_ROWS = struct.Struct("@Q3q")
_CHUNK = _Packed("@4I3QIf" + "Q3q" * 4 + "6Q")
_EVICTION = _Packed("@7I4x6QQ2QQQ")
_NO_ROWS = (0, 0, 0, 0)


def make_score_mods(*, causal=False, scale=0.0, cap=0.0, slopes=None, table=None, doc=None, prefix=None) -> ScoreMods:
    """llmcache_score_mods.  slopes f32 [heads]; table f32 [heads, 2 * reach + 1]; doc i32 [n_seqs, seq_len];
    prefix i32 [n_seqs].  The struct keeps the tensors alive."""
    _dense(slopes, torch.float32, 1, "slopes", True)
    _dense(table, torch.float32, 2, "table", True)
    _dense(doc, torch.int32, 2, "doc", True)
    _dense(prefix, torch.int32, 1, "prefix", True)
    m = ScoreMods()
    m.struct_size = C.sizeof(ScoreMods)
    m.causal, m.scale, m.cap = int(causal), scale, cap
    if table is not None:
        if table.shape[1] % 2 == 0:
            raise LLMCacheError(ERR_SHAPE, "table: an odd number of distances, from -reach to reach")
        m.reach = table.shape[1] // 2
    if doc is not None and prefix is not None and doc.shape[0] != prefix.shape[0]:
        raise LLMCacheError(ERR_SHAPE, "doc and prefix: as many sequences in one as in the other")
    masks = doc if doc is not None else prefix
    m.mask_seqs = 0 if masks is None else masks.shape[0]
    m.slopes, m.table, m.doc, m.prefix = _ptr(slopes), _ptr(table), _ptr(doc), _ptr(prefix)
    m.tensors = (slopes, table, doc, prefix)
    return m


def _same_device(device, *tensors):
    for t in tensors:
        if t is not None and t.get_device() != device:
            _other_device(t, device)


def _check_mods(mods, heads, device, S=0, n=0, layer_len=0):
    """The shapes of the modifiers' arrays (S, n: of whole sequences; layer_len: of a layer, for any number of them)."""
    slopes, table, doc, prefix = tensors = getattr(mods, "tensors", (None, None, None, None))
    _same_device(device, *tensors)
    if (slopes is not None and slopes.size(0) != heads) or (table is not None and table.size(0) != heads):
        raise LLMCacheError(ERR_SHAPE, "score modifiers: one row per query head")
    if S and ((doc is not None and doc.shape != (S, n)) or (prefix is not None and prefix.shape != (S,))):
        raise LLMCacheError(ERR_SHAPE, "doc: [n_seqs, seq_len], prefix: [n_seqs]")
    if layer_len and ((doc is not None and (doc.size(0) == 0 or doc.size(1) != layer_len)) or (prefix is not None and prefix.size(0) == 0)):
        raise LLMCacheError(ERR_SHAPE, "doc: [n_seqs, seq_len of the layer], prefix: [n_seqs], of one sequence at least")


def llmcache_attention(q, k, v, out, mods: Optional[ScoreMods] = None, lse=None, n_seqs_dev=None, stream=None) -> None:
    """out = softmax(modified q k^T) v.  q, out: bf16 [n_seqs, seq_len, heads, 64]; k, v: [n_seqs, seq_len, kv_heads, 64],
    views of any strides (multiples of 8); lse: optional f32 [n_seqs, seq_len, heads]."""
    if not isinstance(q, torch.Tensor) or not isinstance(k, torch.Tensor):
        raise LLMCacheError(ERR_ARG, "llmcache_attention: q and k are tensors")
    device, shape, kv = q.get_device(), q.shape, k.shape
    rq, rk = _rows(q, "q", 4, None, device), _rows(k, "k", 4, None, device)
    S, n, H, _ = shape
    if kv[0] != S or kv[1] != n:
        raise LLMCacheError(ERR_SHAPE, "llmcache_attention: q, out [S, n, H, 64], k, v [S, n, HK, 64]")
    rv, ro = _rows(v, "v", 4, kv, device), _rows(out, "out", 4, shape, device)
    lse_at = _addr(lse, torch.float32, (S, n, H), "lse", device)
    if n_seqs_dev is not None and isinstance(n_seqs_dev, torch.Tensor):
        _same_device(device, n_seqs_dev)
    if mods is not None:
        _check_mods(mods, H, device, S, n)
    pack = _ROWS.pack
    _check(lib().llmcache_attention(pack(*rq), pack(*rk), pack(*rv), pack(*ro), S, n, H, kv[2], _ptr(n_seqs_dev),
                                    C.addressof(mods) if mods is not None else None, lse_at or None, _stream(stream)),
           "llmcache_attention")


def llmcache_attention_status() -> int:
    return int(lib().llmcache_attention_status())


def llmcache_attention_debug_knobs(wait_limit_ns: int, flags: int) -> None:
    _check(lib().llmcache_attention_debug_knobs(wait_limit_ns, flags), "llmcache_attention_debug_knobs")


def llmcache_kv_bytes(desc: KVDesc) -> int:
    out = C.c_size_t(0)
    _check(lib().llmcache_kv_bytes(C.byref(desc), C.byref(out)), "llmcache_kv_bytes")
    return int(out.value)


def llmcache_kv_create(desc: KVDesc) -> int:
    out = C.c_void_p(None)
    _check(lib().llmcache_kv_create(C.byref(desc), C.byref(out)), "llmcache_kv_create")
    return out.value


def llmcache_kv_destroy(kv: int) -> None:
    _check(lib().llmcache_kv_destroy(kv), "llmcache_kv_destroy")


def llmcache_kv_attention(kv, chunk: KVChunk, stream=None) -> None:
    _check(lib().llmcache_kv_attention(kv, C.byref(chunk), _stream(stream)), "llmcache_kv_attention")


def llmcache_kv_evict(kv, eviction: KVEviction, stream=None) -> None:
    _check(lib().llmcache_kv_evict(kv, C.byref(eviction), _stream(stream)), "llmcache_kv_evict")


def llmcache_kv_status(kv) -> int:
    return int(lib().llmcache_kv_status(kv))


def llmcache_kv_debug_knobs(kv, wait_limit_ns: int, flags: int) -> None:
    _check(lib().llmcache_kv_debug_knobs(kv, wait_limit_ns, flags), "llmcache_kv_debug_knobs")


def llmcache_layer_score_mods(layer, mods: Optional[ScoreMods]) -> None:
    _check(lib().llmcache_layer_score_mods(layer, C.byref(mods) if mods is not None else None), "llmcache_layer_score_mods")


def llmcache_layer_extend(layer, kv, x, chunk: KVChunk, out, stream=None) -> None:
    _check(lib().llmcache_layer_extend(layer, kv, _ptr(x), C.byref(chunk), _ptr(out), _stream(stream)), "llmcache_layer_extend")


def make_kv_desc(k_pages, v_pages, *, heads, max_seqs, max_rows, max_len, device=0, workspace=None) -> KVDesc:
    """k_pages, v_pages: bf16 [num_pages, kv_heads, page_size, 64], dense within a page, equal strides between pages."""
    _want(k_pages, torch.bfloat16, 4, "k_pages")
    _want(v_pages, torch.bfloat16, 4, "v_pages")
    num, hk, ps, dh = k_pages.shape
    if v_pages.shape != k_pages.shape or dh != 64 or k_pages.stride() != v_pages.stride() or \
            k_pages.stride()[1:] != (ps * 64, 64, 1):
        raise LLMCacheError(ERR_SHAPE, "k_pages, v_pages: [num_pages, kv_heads, page_size, 64], dense within a page")
    d = KVDesc()
    d.struct_size, d.device = C.sizeof(KVDesc), device
    d.heads, d.kv_heads, d.num_pages, d.page_size = heads, hk, num, ps
    d.max_seqs, d.max_rows, d.max_len = max_seqs, max_rows, max_len
    d.k_pages, d.v_pages, d.page_stride = k_pages.data_ptr(), v_pages.data_ptr(), k_pages.stride(0)
    if workspace is not None:
        d.workspace, d.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    return d


_CHUNK_BYTES = C.sizeof(KVChunk)


class KVCache:
    """Owner of one llmcache_kv_t handle; keeps the page tensors alive (the library borrows them)."""

    def __init__(self, k_pages, v_pages, *, heads, max_seqs, max_rows, max_len, device=None, workspace=None):
        self.k_pages, self.v_pages, self.workspace = k_pages, v_pages, workspace
        self.desc = make_kv_desc(k_pages, v_pages, heads=heads, max_seqs=max_seqs, max_rows=max_rows, max_len=max_len,
                                 device=(k_pages.device.index or 0) if device is None else device, workspace=workspace)
        self.heads, self.kv_heads, self.device = heads, self.desc.kv_heads, self.desc.device
        _same_device(self.device, k_pages, v_pages, workspace)
        self.handle = llmcache_kv_create(self.desc)

    def _pack_chunk(self, n_rows, cu_rows, lens, pages, longest, weights, decay, positions, first, q=_NO_ROWS, out=_NO_ROWS,
                    k_new=_NO_ROWS, v_new=_NO_ROWS, lse=0, mods=None) -> bytes:
        """A llmcache_kv_chunk."""
        device = self.device
        if lens is None or pages is None or cu_rows is None:
            raise LLMCacheError(ERR_ARG, "cu_rows, lens and pages are needed")
        lens_at = _addr(lens, torch.int32, (-1,), "lens", device)
        S = lens.shape[0]
        pages_at = _addr(pages, torch.int32, (S, -1), "pages", device)
        side_ld = w_at = p_at = 0
        if weights is not None:
            w_at, side_ld = _addr(weights, torch.float32, (S, self.kv_heads, -1), "weights", device), weights.shape[-1]
        if positions is not None:
            p_at = _addr(positions, torch.int32, (S, self.kv_heads, side_ld if weights is not None else -1), "positions", device)
            side_ld = positions.shape[-1]
        return _CHUNK(_CHUNK_BYTES, S, n_rows, longest, _addr(cu_rows, torch.int32, (S + 1,), "cu_rows", device), lens_at, pages_at,
                           pages.shape[1], decay if weights is not None else 0.0, *q, *out, *k_new, *v_new, lse, w_at, p_at,
                           _addr(first, torch.int32, (S,), "first", device), side_ld, 0 if mods is None else C.addressof(mods))

    def chunk(self, n_rows, *, cu_rows, lens, pages, longest=0, weights=None, decay=1.0, positions=None, first=None) -> KVChunk:
        """What llmcache_kv_attention and llmcache_layer_extend take alike."""
        return KVChunk.from_buffer_copy(self._pack_chunk(n_rows, cu_rows, lens, pages, longest, weights, decay, positions, first))

    def attention(self, q, out, *, cu_rows, lens, pages, longest=0, k_new=None, v_new=None, lse=None, mods=None, weights=None,
                  decay=1.0, positions=None, first=None, stream=None):
        """Stores k_new, v_new [n_rows, kv_heads, 64] in the pages and lets q [n_rows, heads, 64] attend to all that its
        sequences have there (llmcache_kv_attention).  cu_rows i32 [n_seqs + 1], lens i32 [n_seqs], pages i32
        [n_seqs, pages]; lse f32 [n_rows, heads]; weights f32 and positions i32 [n_seqs, kv_heads, slots].  longest: most rows
        of one sequence (0: not known); its rows beyond that are stored, but out and lse stay as they were there."""
        device = self.device
        rq = _rows(q, "q", 3, None, device)
        T = q.shape[0]
        ro = _rows(out, "out", 3, (T, self.heads, 64), device)
        if q.shape[1] != self.heads:
            raise LLMCacheError(ERR_SHAPE, "q, out: [n_rows, heads, 64]")
        if (k_new is None) != (v_new is None):
            raise LLMCacheError(ERR_ARG, "k_new and v_new come together")
        rk = rv = _NO_ROWS
        if k_new is not None:
            new = (T, self.kv_heads, 64)
            rk, rv = _rows(k_new, "k_new", 3, new, device), _rows(v_new, "v_new", 3, new, device)
        if mods is not None:
            _check_mods(mods, self.heads, device)
        c = self._pack_chunk(T, cu_rows, lens, pages, longest, weights, decay, positions, first, rq, ro, rk, rv,
                             _addr(lse, torch.float32, (T, self.heads), "lse", device), mods)
        _check(lib().llmcache_kv_attention(self.handle, c, _stream(stream, device)), "llmcache_kv_attention")

    def evict(self, *, lens, pages, weights, new_pages, new_lens, budget, recent=0, sinks=0, positions=None, new_weights=None,
              new_positions=None, kept=None, stream=None):
        """Copies the `budget` entries per sequence and head that received the most attention, the newest and the first ones
        to new_pages (llmcache_kv_evict)."""
        device, HK = self.device, self.kv_heads
        I32, F32 = torch.int32, torch.float32
        if lens is None or pages is None or weights is None or new_pages is None or new_lens is None:
            raise LLMCacheError(ERR_ARG, "lens, pages, weights, new_pages and new_lens are needed")
        lens_at = _addr(lens, I32, (-1,), "lens", device)
        S = lens.shape[0]
        pages_at, w_at = _addr(pages, I32, (S, -1), "pages", device), _addr(weights, F32, (S, HK, -1), "weights", device)
        fresh_at, ld = _addr(new_pages, I32, (S, -1), "new_pages", device), weights.shape[2]
        new_w = _addr(new_weights, F32, (S, HK, -1), "new_weights", device)
        new_ld = -1 if new_weights is None else new_weights.shape[2]
        new_p = _addr(new_positions, I32, (S, HK, new_ld), "new_positions", device)
        if new_positions is not None:
            new_ld = new_positions.shape[2]
        e = _EVICTION(_EVICTION.size, S, budget, recent, sinks, pages.shape[1], new_pages.shape[1], lens_at, pages_at, fresh_at,
                           _addr(new_lens, I32, (S,), "new_lens", device), w_at, _addr(positions, I32, (S, HK, ld), "positions", device),
                           ld, new_w, new_p, max(new_ld, 0), _addr(kept, I32, (S, HK, budget), "kept", device))
        _check(lib().llmcache_kv_evict(self.handle, e, _stream(stream, device)), "llmcache_kv_evict")

    def status(self) -> int:
        return llmcache_kv_status(self.handle)

    def debug_knobs(self, wait_limit_ns: int = 0, flags: int = 0):
        llmcache_kv_debug_knobs(self.handle, wait_limit_ns, flags)

    def close(self):
        if getattr(self, "handle", None):
            llmcache_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
