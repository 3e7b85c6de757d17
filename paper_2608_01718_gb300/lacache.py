"""Python binding of liblacache.so (include/lacache.h): the same entry points under the same names.

Argument marshalling only. Tensors are passed by their data pointers; ``cuda_stream`` defaults to torch's current
stream on the handle's device. Every step of the lookup runs in the library's CUDA kernels. There is no CPU path:
if the library has not been built, loading it raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_build", "liblacache.so")

LACACHE_OK, LACACHE_ERR_INVALID_ARG, LACACHE_ERR_CAPACITY, LACACHE_ERR_OOM = 0, 1, 2, 3
LACACHE_ERR_CUDA, LACACHE_ERR_DEVICE_TIMEOUT, LACACHE_ERR_UNSUPPORTED, LACACHE_ERR_IO = 4, 5, 6, 7
LACACHE_CHECK_EMB, LACACHE_CHECK_TOKENS, LACACHE_CHECK_BOTH = 0, 1, 2
LACACHE_BF16, LACACHE_F32, LACACHE_F16 = 0, 1, 2
LACACHE_STAGE1_AUTO, LACACHE_STAGE1_TENSOR, LACACHE_STAGE1_STREAM, LACACHE_STAGE1_LSH = 0, 1, 2, 3
LACACHE_STAGE1_TENSOR_PAIR = 4   # reported by lacache_last_launch only
LACACHE_STAGE1_LSH_TENSOR = 5    # reported by lacache_last_launch only
LACACHE_MISS_KEY, LACACHE_HIT, LACACHE_REJECT = 0, 1, 2

LACACHE_ROPE_HALF, LACACHE_ROPE_INTERLEAVED = 0, 1
LACACHE_ROPE_PLAIN, LACACHE_ROPE_LINEAR, LACACHE_ROPE_BASE, LACACHE_ROPE_BANDED = 0, 1, 2, 3
LACACHE_KV_BF16, LACACHE_KV_F16, LACACHE_KV_E4M3, LACACHE_KV_INT8 = 0, 1, 2, 3

LACACHE_MAX_MODELS = 8
LACACHE_MAX_SHARDS = 16
LACACHE_MAX_HEAD_DIM = 256

EXPORTS = ["lacache_create", "lacache_create_ensemble", "lacache_destroy", "lacache_insert", "lacache_lookup",
           "lacache_lookup_host", "lacache_lookup_host_async", "lacache_append_misses", "lacache_read_rows",
           "lacache_size", "lacache_sync", "lacache_last_launch", "lacache_stage_timing", "lacache_stage_times",
           "lacache_inject_stall", "lacache_enable_lsh", "lacache_read_signatures", "lacache_calibrate",
           "lacache_calibrate_workspace_bytes", "lacache_verify_draft", "lacache_lookup_noalloc",
           "lacache_merge_shards", "lacache_get_stats", "lacache_save", "lacache_load", "lacache_get_config",
           "lacache_rope_init", "lacache_rope_apply", "lacache_kv_create", "lacache_kv_destroy", "lacache_kv_get_pool",
           "lacache_kv_append", "lacache_kv_read", "lacache_kv_attend", "lacache_kv_sync", "lacache_kv_inject_stall",
           "lacache_status_string"]


class lacache_config(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("k", ctypes.c_int32), ("capacity", ctypes.c_int64),
                ("tau_c", ctypes.c_float), ("tau_a", ctypes.c_float), ("top_c", ctypes.c_int32),
                ("token_match_min", ctypes.c_int32), ("check_mode", ctypes.c_int32), ("max_batch", ctypes.c_int32),
                ("device", ctypes.c_int32), ("stage1", ctypes.c_int32)]


class lacache_ensemble(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int32), ("dims", ctypes.c_int32 * LACACHE_MAX_MODELS),
                ("tau_a", ctypes.c_float * LACACHE_MAX_MODELS)]


class lacache_result(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in
                ("entry_id", "status", "key_score", "prefix_score", "token_matches", "n_cand",
                 "cand_id", "cand_score", "cand_prefix_score", "cand_matches", "prefix_scores", "cand_pass",
                 "cand_prefix_scores")]


class lacache_stats(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int64) for name in
                ("lookups", "queries", "hits", "rejects", "key_misses", "inserted", "appended")]


class lacache_shard_result(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in
                ("cand_id", "cand_score", "cand_prefix_score", "cand_matches", "cand_pass", "cand_prefix_scores",
                 "key_score", "n_cand")] + [("id_base", ctypes.c_int64)]


class lacache_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class lacache_rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("amplitude", ctypes.c_float),
                ("reserved", ctypes.c_int32), ("turn", ctypes.c_uint64 * (LACACHE_MAX_HEAD_DIM // 2))]


class lacache_kv_config(ctypes.Structure):
    _fields_ = [("layers", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("pages", ctypes.c_int64), ("format", ctypes.c_int32),
                ("device", ctypes.c_int32)]


class lacache_kv_pool(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("k", "v", "k_scale", "v_scale")]


class lacache_kv_table(ctypes.Structure):
    _fields_ = [("pages_dev", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("seqs", ctypes.c_int32),
                ("width", ctypes.c_int32)]


class lacache_attention(ctypes.Structure):
    _fields_ = [("new_tokens", ctypes.c_int32), ("q_heads", ctypes.c_int32), ("window", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("lengths_dev", ctypes.c_void_p),
                ("starts_dev", ctypes.c_void_p), ("q", lacache_rows), ("out", lacache_rows),
                ("lse_dev", ctypes.c_void_p)]


class LacacheError(RuntimeError):
    def __init__(self, call: str, status: int):
        super().__init__(f"{call}: {status_string(status)} ({status})")
        self.status = status


_lib = None


def load() -> ctypes.CDLL:
    """Open liblacache.so (once). Raises if it has not been built: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_01718_gb300.build` "
                           "(or __graft_entry__.build()); the lookup has no CPU fallback")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    p64 = ctypes.POINTER(ctypes.c_int64)
    p32 = ctypes.POINTER(ctypes.c_int32)
    sig = {
        "lacache_create": ([ctypes.POINTER(lacache_config), ctypes.POINTER(vp)], i32),
        "lacache_create_ensemble": ([ctypes.POINTER(lacache_config), ctypes.POINTER(lacache_ensemble),
                                     ctypes.POINTER(vp)], i32),
        "lacache_destroy": ([vp], i32),
        "lacache_insert": ([vp, i64, vp, vp, vp, i32, p64, vp], i32),
        "lacache_lookup": ([vp, i32, vp, vp, vp, ctypes.POINTER(lacache_result), vp], i32),
        "lacache_lookup_host": ([vp, i32, vp, vp, vp, ctypes.POINTER(lacache_result), vp], i32),
        "lacache_lookup_host_async": ([vp, i32, vp, vp, vp, ctypes.POINTER(lacache_result), vp], i32),
        "lacache_append_misses": ([vp, i32, vp, vp, vp, vp, p64, p64, vp], i32),
        "lacache_read_rows": ([vp, i64, i64, vp, vp, vp, vp], i32),
        "lacache_size": ([vp, p64], i32),
        "lacache_sync": ([vp], i32),
        "lacache_last_launch": ([vp, p32, p32], i32),
        "lacache_stage_timing": ([vp, i32], i32),
        "lacache_stage_times": ([vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), p64], i32),
        "lacache_inject_stall": ([vp, i32], i32),
        "lacache_enable_lsh": ([vp, i32, i32, vp, vp], i32),
        "lacache_read_signatures": ([vp, i64, i64, vp, vp], i32),
        "lacache_calibrate": ([i64, i32, vp, vp, ctypes.c_double, ctypes.c_float, vp, vp, vp, vp], i32),
        "lacache_calibrate_workspace_bytes": ([], ctypes.c_size_t),
        "lacache_verify_draft": ([i32, i32, vp, vp, vp, vp, vp], i32),
        "lacache_lookup_noalloc": ([ctypes.POINTER(lacache_config), i64, vp, vp, vp, i32, vp, vp, vp,
                                    ctypes.POINTER(lacache_result), vp], i32),
        "lacache_get_stats": ([vp, ctypes.POINTER(lacache_stats), i32], i32),
        "lacache_save": ([vp, ctypes.c_char_p], i32),
        "lacache_load": ([ctypes.c_char_p, i32, i64, ctypes.POINTER(vp)], i32),
        "lacache_get_config": ([vp, ctypes.POINTER(lacache_config), ctypes.POINTER(lacache_ensemble)], i32),
        "lacache_merge_shards": ([i32, ctypes.POINTER(lacache_shard_result), i32, i32, i32,
                                  ctypes.POINTER(lacache_result), vp], i32),
        "lacache_rope_init": ([i32, i32, ctypes.c_double, i32, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                               ctypes.c_double, ctypes.c_float, ctypes.POINTER(lacache_rope)], i32),
        "lacache_rope_apply": ([vp, i64, i32, i32, i32, vp, vp, i32, vp, vp], i32),
        "lacache_kv_create": ([ctypes.POINTER(lacache_kv_config), ctypes.POINTER(vp)], i32),
        "lacache_kv_destroy": ([vp], i32),
        "lacache_kv_get_pool": ([vp, i32, ctypes.POINTER(lacache_kv_pool)], i32),
        "lacache_kv_append": ([vp, i32, vp, i64, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp], i32),
        "lacache_kv_read": ([vp, i32, vp, i64, vp, vp, i32, vp, vp, vp], i32),
        "lacache_kv_attend": ([vp, i32, vp, vp, vp], i32),
        "lacache_kv_sync": ([vp], i32),
        "lacache_kv_inject_stall": ([vp, i32], i32),
        "lacache_status_string": ([i32], ctypes.c_char_p),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().lacache_status_string(int(status)).decode()


def _check(call: str, status: int) -> None:
    if status != LACACHE_OK:
        raise LacacheError(call, status)


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(cuda_stream, device: int | None = None):
    if cuda_stream is not None:
        return cuda_stream if isinstance(cuda_stream, int) else cuda_stream.cuda_stream
    import torch
    return torch.cuda.current_stream(device).cuda_stream


def _results_on(cuda_stream, device):
    """Where a call's results are allocated: from the memory of the stream that the call runs on. (A block of another stream's
    may still be in use there by work that was queued before the block was freed.)"""
    if cuda_stream is None:
        return contextlib.nullcontext()
    import torch
    if isinstance(cuda_stream, int):   # 0 is the default stream
        cuda_stream = torch.cuda.ExternalStream(cuda_stream, device) if cuda_stream else torch.cuda.default_stream(device)
    return torch.cuda.stream(cuda_stream)


def make_config(d: int, k: int, capacity: int, tau_c: float, tau_a: float, top_c: int, *, max_batch: int,
                check_mode: int = LACACHE_CHECK_EMB, token_match_min: int = 0, device: int = 0,
                stage1: int = LACACHE_STAGE1_AUTO) -> lacache_config:
    return lacache_config(d, k, capacity, tau_c, tau_a, top_c, token_match_min, check_mode, max_batch, device, stage1)


def lacache_create(cfg: lacache_config) -> int:
    h = ctypes.c_void_p()
    _check("lacache_create", load().lacache_create(ctypes.byref(cfg), ctypes.byref(h)))
    return h.value


def make_ensemble(dims, taus) -> lacache_ensemble:
    ens = lacache_ensemble()
    ens.m = len(dims)
    for i, (d, t) in enumerate(zip(dims, taus)):
        ens.dims[i] = d
        ens.tau_a[i] = t
    return ens


def lacache_create_ensemble(cfg: lacache_config, ens: lacache_ensemble) -> int:
    h = ctypes.c_void_p()
    _check("lacache_create_ensemble", load().lacache_create_ensemble(ctypes.byref(cfg), ctypes.byref(ens),
                                                                     ctypes.byref(h)))
    return h.value


def lacache_destroy(h: int) -> None:
    _check("lacache_destroy", load().lacache_destroy(h))


def lacache_insert(h: int, key, prefix, ids, dtype: int = LACACHE_BF16, cuda_stream=None) -> int:
    """Append rows (device tensors [n x d], [n x d], [n x k] int32); returns the first new entry id."""
    first = ctypes.c_int64()
    n = int(ids.shape[0])
    _check("lacache_insert", load().lacache_insert(h, n, _ptr(key), _ptr(prefix), _ptr(ids), dtype,
                                                   ctypes.byref(first), _stream(cuda_stream)))
    return first.value


def _result_struct(out: dict) -> lacache_result:
    return lacache_result(*[_ptr(out.get(name)) for name, _ in lacache_result._fields_])


def lacache_lookup(h: int, q_emb, q_prefix, q_ids, out: dict, cuda_stream=None) -> None:
    """Batched lookup; ``out`` maps lacache_result field names to caller-owned device tensors."""
    res = _result_struct(out)
    _check("lacache_lookup", load().lacache_lookup(h, int(q_emb.shape[0]), _ptr(q_emb), _ptr(q_prefix),
                                                   _ptr(q_ids), ctypes.byref(res), _stream(cuda_stream)))


def lacache_get_stats(h: int, reset: bool = False) -> dict:
    """The handle's decision counters (synchronizes its device); reset zeroes them after reading."""
    st = lacache_stats()
    _check("lacache_get_stats", load().lacache_get_stats(h, ctypes.byref(st), int(reset)))
    return {name: int(getattr(st, name)) for name, _ in lacache_stats._fields_}


def lacache_save(h: int, path: str) -> None:
    """Write the cache (configuration and valid entries) to ``path``."""
    _check("lacache_save", load().lacache_save(h, os.fsencode(path)))


def lacache_load(path: str, device: int = 0, capacity: int = 0) -> int:
    """A new handle on ``device`` from a saved cache; capacity > 0 replaces the saved capacity."""
    h = ctypes.c_void_p()
    _check("lacache_load", load().lacache_load(os.fsencode(path), device, capacity, ctypes.byref(h)))
    return h.value


def lacache_get_config(h: int) -> tuple:
    """(lacache_config, lacache_ensemble) of a handle."""
    cfg, ens = lacache_config(), lacache_ensemble()
    _check("lacache_get_config", load().lacache_get_config(h, ctypes.byref(cfg), ctypes.byref(ens)))
    return cfg, ens


def lacache_merge_shards(shards: list, top_c: int, models: int, out: dict, cuda_stream=None) -> None:
    """Merge entry-range shards' lookup outputs (``shards``: one (outputs dict, id_base) per shard, outputs as
    alloc_result(candidates=True) writes them) into ``out``, the whole-store result."""
    arr = (lacache_shard_result * len(shards))()
    for g, (o, base) in enumerate(shards):
        arr[g] = lacache_shard_result(*[_ptr(o.get(name)) for name, _ in lacache_shard_result._fields_[:-1]],
                                      int(base))
    res = _result_struct(out)
    B = int(out["status"].shape[0])
    _check("lacache_merge_shards", load().lacache_merge_shards(len(shards), arr, B, top_c, models, ctypes.byref(res),
                                                               _stream(cuda_stream)))


def lacache_lookup_host(h: int, q_emb, q_prefix, q_ids, out: dict, cuda_stream=None) -> None:
    """Lookup of host-resident queries into host-resident results (synchronous)."""
    res = _result_struct(out)
    _check("lacache_lookup_host", load().lacache_lookup_host(h, int(q_emb.shape[0]), _ptr(q_emb), _ptr(q_prefix),
                                                             _ptr(q_ids), ctypes.byref(res), _stream(cuda_stream)))


def lacache_lookup_host_async(h: int, q_emb, q_prefix, q_ids, out: dict, cuda_stream=None) -> None:
    """Lookup of queries in pinned host tensors into pinned host results, enqueued on the stream without waiting:
    the results are there once the stream has passed the call."""
    res = _result_struct(out)
    _check("lacache_lookup_host_async", load().lacache_lookup_host_async(
        h, int(q_emb.shape[0]), _ptr(q_emb), _ptr(q_prefix), _ptr(q_ids), ctypes.byref(res), _stream(cuda_stream)))


def lacache_append_misses(h: int, q_emb, q_prefix, q_ids, status, cuda_stream=None) -> tuple[int, int]:
    """Append every non-HIT query of a looked-up batch in query order; returns (first id, count)."""
    first, n = ctypes.c_int64(), ctypes.c_int64()
    _check("lacache_append_misses", load().lacache_append_misses(
        h, int(q_emb.shape[0]), _ptr(q_emb), _ptr(q_prefix), _ptr(q_ids), _ptr(status), ctypes.byref(first),
        ctypes.byref(n), _stream(cuda_stream)))
    return first.value, n.value


def lacache_read_rows(h: int, first: int, n: int, key=None, prefix=None, ids=None, cuda_stream=None) -> None:
    _check("lacache_read_rows", load().lacache_read_rows(h, first, n, _ptr(key), _ptr(prefix), _ptr(ids),
                                                         _stream(cuda_stream)))


def lacache_size(h: int) -> int:
    n = ctypes.c_int64()
    _check("lacache_size", load().lacache_size(h, ctypes.byref(n)))
    return n.value


def lacache_sync(h: int) -> None:
    _check("lacache_sync", load().lacache_sync(h))


def lacache_last_launch(h: int) -> tuple[int, int]:
    splits, kernel = ctypes.c_int32(), ctypes.c_int32()
    _check("lacache_last_launch", load().lacache_last_launch(h, ctypes.byref(splits), ctypes.byref(kernel)))
    return splits.value, kernel.value


def lacache_stage_timing(h: int, max_lookups: int) -> None:
    _check("lacache_stage_timing", load().lacache_stage_timing(h, max_lookups))


def lacache_stage_times(h: int) -> tuple[float, float, int]:
    """(stage-1 ms, stage-2 ms, lookups timed) summed since the previous call."""
    t1, t2, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int64()
    _check("lacache_stage_times", load().lacache_stage_times(h, ctypes.byref(t1), ctypes.byref(t2), ctypes.byref(n)))
    return t1.value, t2.value, n.value


def lacache_inject_stall(h: int, lookups: int) -> None:
    _check("lacache_inject_stall", load().lacache_inject_stall(h, lookups))


def lacache_enable_lsh(h: int, bits: int, radius: int, hyperplanes, cuda_stream=None) -> None:
    """Build the SimHash index: signatures of every entry against hyperplanes ([bits x d] bf16)."""
    _check("lacache_enable_lsh", load().lacache_enable_lsh(h, bits, radius, _ptr(hyperplanes), _stream(cuda_stream)))


def lacache_read_signatures(h: int, first: int, n: int, out, cuda_stream=None) -> None:
    _check("lacache_read_signatures", load().lacache_read_signatures(h, first, n, _ptr(out), _stream(cuda_stream)))


def lacache_calibrate_workspace_bytes() -> int:
    return int(load().lacache_calibrate_workspace_bytes())


def lacache_calibrate(x, y, percentile: float, cap: float, sims, result, workspace, cuda_stream=None) -> None:
    """Pair similarities of (x_i, y_i) into sims, then result = [nearest-rank percentile, min(cap, it)]."""
    _check("lacache_calibrate", load().lacache_calibrate(int(x.shape[0]), int(x.shape[1]), _ptr(x), _ptr(y),
                                                         float(percentile), float(cap), _ptr(sims), _ptr(result),
                                                         _ptr(workspace), _stream(cuda_stream)))


def lacache_verify_draft(p_target, p_draft, status, accepted, cuda_stream=None) -> None:
    """Accepted draft-prefix length per query (P_f >= P_g from the first token on); -1 for served queries."""
    B, k = int(p_target.shape[0]), int(p_target.shape[1])
    _check("lacache_verify_draft", load().lacache_verify_draft(B, k, _ptr(p_target), _ptr(p_draft), _ptr(status),
                                                               _ptr(accepted), _stream(cuda_stream)))


def lacache_lookup_noalloc(cfg: lacache_config, key, prefix, ids, q_emb, q_prefix, q_ids, out: dict,
                           cuda_stream=None) -> None:
    """Lookup against caller-owned cache rows with no device allocation (see include/lacache.h)."""
    res = _result_struct(out)
    n = int(ids.shape[0]) if ids is not None else 0
    _check("lacache_lookup_noalloc", load().lacache_lookup_noalloc(
        ctypes.byref(cfg), n, _ptr(key), _ptr(prefix), _ptr(ids), int(q_emb.shape[0]), _ptr(q_emb),
        _ptr(q_prefix), _ptr(q_ids), ctypes.byref(res), _stream(cuda_stream, cfg.device)))


def lacache_rope_init(rot_dim: int, layout: int = LACACHE_ROPE_HALF, base: float = 10000.0,
                      scaling: int = LACACHE_ROPE_PLAIN, factor: float = 1.0, original_len: float = 0.0,
                      low_turns: float = 1.0, high_turns: float = 4.0, amplitude: float = 1.0) -> lacache_rope:
    """The plan of a rotation (host only)."""
    rope = lacache_rope()
    _check("lacache_rope_init", load().lacache_rope_init(rot_dim, layout, base, scaling, factor, original_len, low_turns,
                                                         high_turns, amplitude, ctypes.byref(rope)))
    return rope


def lacache_rope_apply(rope, n: int, heads: int, head_dim: int, dtype: int, x: lacache_rows, pos, inverse: bool,
                       y: lacache_rows, cuda_stream=None) -> None:
    """Rotate n x heads rows (lacache_rows of device memory) at the positions ``pos`` (int32 on the device)."""
    _check("lacache_rope_apply", load().lacache_rope_apply(ctypes.addressof(rope), n, heads, head_dim, dtype,
                                                           ctypes.addressof(x), _ptr(pos), int(inverse),
                                                           ctypes.addressof(y), _stream(cuda_stream)))


def _address(struct) -> int | None:
    return None if struct is None else ctypes.addressof(struct)


def lacache_kv_create(cfg: lacache_kv_config) -> int:
    h = ctypes.c_void_p()
    _check("lacache_kv_create", load().lacache_kv_create(ctypes.byref(cfg), ctypes.byref(h)))
    return h.value


def lacache_kv_destroy(h: int) -> None:
    _check("lacache_kv_destroy", load().lacache_kv_destroy(h))


def lacache_kv_get_pool(h: int, layer: int = 0) -> lacache_kv_pool:
    pool = lacache_kv_pool()
    _check("lacache_kv_get_pool", load().lacache_kv_get_pool(h, layer, ctypes.byref(pool)))
    return pool


def lacache_kv_append(h: int, layer: int, table: lacache_kv_table, n: int, seq, pos, rope, rope_pos, dtype: int,
                      k: lacache_rows, v: lacache_rows, q_heads: int = 0, q: lacache_rows | None = None,
                      q_out: lacache_rows | None = None, cuda_stream=None) -> None:
    """Write n tokens into the cache (rope: a lacache_rope or None; q and q_out: rows rotated with k, or None)."""
    _check("lacache_kv_append", load().lacache_kv_append(
        h, layer, _address(table), n, _ptr(seq), _ptr(pos), _address(rope), _ptr(rope_pos), dtype, _address(k),
        _address(v), q_heads, _address(q), _address(q_out), _stream(cuda_stream)))


def lacache_kv_read(h: int, layer: int, table: lacache_kv_table, n: int, seq, pos, dtype: int, k: lacache_rows | None,
                    v: lacache_rows | None, cuda_stream=None) -> None:
    """Read n cached tokens back as rows of ``dtype``."""
    _check("lacache_kv_read", load().lacache_kv_read(h, layer, _address(table), n, _ptr(seq), _ptr(pos), dtype,
                                                     _address(k), _address(v), _stream(cuda_stream)))


def lacache_kv_attend(h: int, layer: int, table: lacache_kv_table, attention: lacache_attention,
                      cuda_stream=None) -> None:
    """Attention of the last new tokens of every sequence over its cached tokens."""
    _check("lacache_kv_attend", load().lacache_kv_attend(h, layer, _address(table), _address(attention),
                                                         _stream(cuda_stream)))


def lacache_kv_sync(h: int) -> None:
    _check("lacache_kv_sync", load().lacache_kv_sync(h))


def lacache_kv_inject_stall(h: int, attends: int) -> None:
    _check("lacache_kv_inject_stall", load().lacache_kv_inject_stall(h, attends))


def alloc_result(batch: int, top_c: int, device, candidates: bool = True, pinned: bool = False,
                 models: int = 0) -> dict:
    """Output buffers of one lookup: device tensors (or pinned host tensors with ``device="cpu"``). ``candidates``
    adds the per-candidate arrays (with their pass bits); ``models`` > 0 adds every model's lookahead scores, for
    the shown candidate and, with ``candidates``, per candidate."""
    import torch
    kw = {"device": device}
    if pinned:
        kw["pin_memory"] = True
    out = {"entry_id": torch.empty(batch, dtype=torch.int32, **kw),
           "status": torch.empty(batch, dtype=torch.uint8, **kw),
           "key_score": torch.empty(batch, dtype=torch.float32, **kw),
           "prefix_score": torch.empty(batch, dtype=torch.float32, **kw),
           "token_matches": torch.empty(batch, dtype=torch.int32, **kw),
           "n_cand": torch.empty(batch, dtype=torch.int32, **kw)}
    if candidates:
        out.update({"cand_id": torch.empty((batch, top_c), dtype=torch.int32, **kw),
                    "cand_score": torch.empty((batch, top_c), dtype=torch.float32, **kw),
                    "cand_prefix_score": torch.empty((batch, top_c), dtype=torch.float32, **kw),
                    "cand_matches": torch.empty((batch, top_c), dtype=torch.int32, **kw),
                    "cand_pass": torch.empty((batch, top_c), dtype=torch.uint8, **kw)})
    if models:
        out["prefix_scores"] = torch.empty((batch, models), dtype=torch.float32, **kw)
        if candidates:
            out["cand_prefix_scores"] = torch.empty((batch, top_c, models), dtype=torch.float32, **kw)
    return out


class LaCache:
    """A handle with its configuration: thin convenience over the functions above."""

    def __init__(self, d: int, k: int, capacity: int, tau_c: float, tau_a: float, top_c: int, *, max_batch: int,
                 check_mode: int = LACACHE_CHECK_EMB, token_match_min: int = 0, device: int = 0,
                 stage1: int = LACACHE_STAGE1_AUTO, prefix_dims=None, tau_a_models=None):
        self.cfg = make_config(d, k, capacity, tau_c, tau_a, top_c, max_batch=max_batch, check_mode=check_mode,
                               token_match_min=token_match_min, device=device, stage1=stage1)
        self.device = device
        self.h = None
        if prefix_dims is None:
            self.models = 1
            self.h = lacache_create(self.cfg)
        else:
            self.models = len(prefix_dims)
            self.h = lacache_create_ensemble(self.cfg, make_ensemble(prefix_dims, tau_a_models))

    @classmethod
    def load(cls, path: str, device: int = 0, capacity: int = 0) -> "LaCache":
        """A cache saved with save(), on ``device``."""
        obj = cls.__new__(cls)
        obj.h = lacache_load(path, device, capacity)
        obj.cfg, ens = lacache_get_config(obj.h)
        obj.device = device
        obj.models = int(ens.m)
        return obj

    def save(self, path: str) -> None:
        lacache_save(self.h, path)

    def close(self) -> None:
        if self.h:
            lacache_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def insert(self, key, prefix, ids, dtype: int = LACACHE_BF16, cuda_stream=None) -> int:
        return lacache_insert(self.h, key, prefix, ids, dtype, cuda_stream)

    def lookup(self, q_emb, q_prefix, q_ids, out: dict | None = None, candidates: bool = True,
               cuda_stream=None) -> dict:
        if out is None:
            with _results_on(cuda_stream, self.device):
                out = alloc_result(q_emb.shape[0], self.cfg.top_c, q_emb.device, candidates, models=self.models)
        lacache_lookup(self.h, q_emb, q_prefix, q_ids, out, cuda_stream)
        return out

    def stats(self, reset: bool = False) -> dict:
        return lacache_get_stats(self.h, reset)

    def append_misses(self, q_emb, q_prefix, q_ids, status, cuda_stream=None) -> tuple[int, int]:
        return lacache_append_misses(self.h, q_emb, q_prefix, q_ids, status, cuda_stream)

    @property
    def size(self) -> int:
        return lacache_size(self.h)

    def sync(self) -> None:
        lacache_sync(self.h)

    def last_launch(self) -> tuple[int, int]:
        return lacache_last_launch(self.h)


# What the calls that decode token by token need of torch, which is imported late: a call's every look-up of it would be a
# tenth of the call.
_DTYPES: dict = {}   # torch dtype -> lacache_dtype
_INT32 = _RAW_STREAM = _Rotation = None


def _bind_torch() -> None:
    global _INT32, _RAW_STREAM, _Rotation
    if _Rotation is not None:
        return
    import torch

    class _Rotation(torch.autograd.Function):
        """Rope.apply for autograd: linear, its gradient the inverse at the same positions."""

        @staticmethod
        def forward(ctx, x, pos, rope, inverse, cuda_stream):
            ctx.save_for_backward(pos)
            ctx.rope, ctx.inverse = rope, inverse
            return rope.apply(x, pos, inverse, cuda_stream=cuda_stream)

        @staticmethod
        def backward(ctx, grad):
            return ctx.rope.apply(grad.contiguous(), ctx.saved_tensors[0], not ctx.inverse), None, None, None, None

    _DTYPES.update({torch.bfloat16: LACACHE_BF16, torch.float16: LACACHE_F16, torch.float32: LACACHE_F32})
    _INT32, _RAW_STREAM = torch.int32, getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _dtype(t) -> int:
    """The lacache_dtype of a tensor's elements."""
    got = _DTYPES.get(t.dtype)
    if got is None:
        raise ValueError(f"rows are bf16, f16 or f32, not {t.dtype}")
    return got


def _current_stream(cuda_stream, device: int) -> int:
    """As _stream, for the calls that decode token by token: torch's raw handle where it offers one (a microsecond less)."""
    if cuda_stream is None and _RAW_STREAM is not None:
        return _RAW_STREAM(device)
    return _stream(cuda_stream, device)


def _new_like(x, cuda_stream, device: int):
    """A dense tensor of x's shape and type for the results of a call on cuda_stream."""
    import torch
    if cuda_stream is None:
        return torch.empty_like(x, memory_format=torch.contiguous_format)
    with _results_on(cuda_stream, device):
        return torch.empty_like(x, memory_format=torch.contiguous_format)


def _rows(name: str, t, n: int, heads: int, head_dim: int, device: int, dtype) -> lacache_rows:
    """A [n x heads x head_dim] CUDA tensor (any strides, dense rows) as lacache_rows."""
    if t.shape != (n, heads, head_dim):
        raise ValueError(f"{name} is [{n} x {heads} x {head_dim}], not {tuple(t.shape)}")
    stride = t.stride()
    if stride[2] != 1 or t.dtype != dtype or t.get_device() != device:
        raise ValueError(f"{name} has dense rows of {dtype} on cuda:{device}")
    return lacache_rows(t.data_ptr(), stride[0], stride[1])


def _index(name: str, t, n: int, device: int) -> int:
    """An int32 [n] CUDA tensor's address."""
    if t.dtype != _INT32 or t.shape != (n,) or not t.is_contiguous() or t.get_device() != device:
        raise ValueError(f"{name} is a dense int32 tensor of {n} on cuda:{device}")
    return t.data_ptr()


def _three(name: str, t):
    if t.dim() != 3 or not t.is_cuda:
        raise ValueError(f"{name} is a [tokens x heads x head_dim] CUDA tensor")
    return t.shape


class Rope:
    """Rotary positions of the first ``rot_dim`` elements of a head: the plan lacache_rope_init makes.

    ``scaling``: None, "linear" (positions divided by ``factor``), "base" (the base stretched so that the slowest pair is) or
    "banded" (only pairs that make few turns within ``original_len`` are stretched)."""

    def __init__(self, rot_dim: int, base: float = 10000.0, interleaved: bool = False, scaling: str | None = None,
                 factor: float = 1.0, original_len: float = 0.0, low_turns: float = 1.0, high_turns: float = 4.0,
                 amplitude: float = 1.0):
        modes = {None: LACACHE_ROPE_PLAIN, "linear": LACACHE_ROPE_LINEAR, "base": LACACHE_ROPE_BASE,
                 "banded": LACACHE_ROPE_BANDED}
        if scaling not in modes:
            raise ValueError(f"scaling is one of {list(modes)}, not {scaling!r}")
        _bind_torch()
        self.plan = lacache_rope_init(rot_dim, LACACHE_ROPE_INTERLEAVED if interleaved else LACACHE_ROPE_HALF, base,
                                      modes[scaling], factor, original_len, low_turns, high_turns, amplitude)

    def apply(self, x, pos, inverse: bool = False, out=None, cuda_stream=None):
        """x [n x heads x head_dim] rotated at ``pos`` (int32 [n]) into ``out`` (new if None; x itself for in place).
        ``inverse``: the transpose, which is the gradient; autograd takes it, where there is no ``out``."""
        n, heads, head_dim = _three("x", x)
        device, dtype = x.get_device(), x.dtype
        import torch
        if (x.requires_grad or out is not None and out.requires_grad) and torch.is_grad_enabled():
            if out is not None:
                raise ValueError("autograd does not follow a rotation into a given out: use torch.no_grad(), or no out")
            return _Rotation.apply(x, pos, self, inverse, cuda_stream)
        if out is None:
            out = _new_like(x, cuda_stream, device)
        args = (self.plan, n, heads, head_dim, _dtype(x), _rows("x", x, n, heads, head_dim, device, dtype),
                _index("pos", pos, n, device), inverse, _rows("out", out, n, heads, head_dim, device, dtype),
                _current_stream(cuda_stream, device))
        if torch.cuda.current_device() == device:
            lacache_rope_apply(*args)
        else:
            with torch.cuda.device(device):
                lacache_rope_apply(*args)
        return out


class _DeviceArray:
    """A view of a handle's device memory for torch.as_tensor (it keeps the handle alive)."""

    def __init__(self, owner, ptr: int, shape, typestr: str):
        self.owner = owner
        self.__cuda_array_interface__ = {"data": (ptr, False), "shape": tuple(shape), "typestr": typestr, "version": 3}


class KVCache:
    """A paged key-value cache (lacache_kv_t) with its calls. ``format``: "bf16", "f16", "e4m3" or "int8".

    Tables are int32 [sequences x pages] CUDA tensors, lengths and positions int32 vectors, rows [tokens x heads x head_dim]
    tensors with dense rows. Calls run on torch's current stream of the cache's device unless given another (and then allocate
    the results that they are not given from its memory). A cache's calls share scratch: issue them on one stream, or order the
    streams by events. Autograd does not follow them."""

    FORMATS = {"bf16": LACACHE_KV_BF16, "f16": LACACHE_KV_F16, "e4m3": LACACHE_KV_E4M3, "int8": LACACHE_KV_INT8}

    def __init__(self, kv_heads: int, head_dim: int, pages: int, page_size: int = 16, format: str = "bf16",
                 layers: int = 1, device: int = 0):
        self.h = None
        if format not in self.FORMATS:
            raise ValueError(f"format is one of {list(self.FORMATS)}, not {format!r}")
        self.cfg = lacache_kv_config(layers, kv_heads, head_dim, page_size, pages, self.FORMATS[format], device)
        self.format, self.device, self.layers = format, device, layers
        _bind_torch()
        self.h, self._lib = lacache_kv_create(self.cfg), load()

    def close(self) -> None:
        if self.h:
            lacache_kv_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _layer(self, layer: int) -> int:   # (ctypes would drop the bits past 32)
        if not 0 <= layer < self.layers:
            raise ValueError(f"layer is 0 to {self.layers - 1}, not {layer}")
        return layer

    def pool(self, layer: int = 0) -> dict:
        """A layer's arrays as tensors on the handle's own memory (valid until close): k and v
        [pages x kv_heads x page_size x head_dim] and, in 8-bit formats, their fp32 scales ks and vs."""
        import torch
        c, p = self.cfg, lacache_kv_get_pool(self.h, self._layer(layer))
        rows = (c.pages, c.kv_heads, c.page_size)
        typestr, dtype = {"bf16": ("<i2", torch.bfloat16), "f16": ("<f2", torch.float16),
                          "e4m3": ("|u1", torch.float8_e4m3fn), "int8": ("|i1", torch.int8)}[self.format]

        def view(ptr, shape, kind):
            return torch.as_tensor(_DeviceArray(self, ptr, shape, kind), device=f"cuda:{self.device}")

        out = {name: view(ptr, (*rows, c.head_dim), typestr).view(dtype) for name, ptr in (("k", p.k), ("v", p.v))}
        if p.k_scale:
            out["ks"], out["vs"] = view(p.k_scale, rows, "<f4"), view(p.v_scale, rows, "<f4")
        return out

    def _table(self, table) -> lacache_kv_table:
        if table.dim() != 2 or table.dtype != _INT32 or table.stride(1) != 1 or table.get_device() != self.device:
            raise ValueError(f"a table is an int32 [sequences x pages] tensor on cuda:{self.device} with dense rows")
        seqs, width = table.shape
        return lacache_kv_table(table.data_ptr(), table.stride(0), seqs, width)

    def append(self, k, v, seq, pos, table, layer: int = 0, rope: Rope | None = None, rope_pos=None, q=None, q_out=None,
               cuda_stream=None):
        """Write k and v [n x kv_heads x head_dim] at positions ``pos`` of sequences ``seq`` (int32 [n]; -1 skips a token),
        k rotated by ``rope`` first. With ``q``, returns it rotated (in ``q_out`` if given)."""
        n, heads, D, dev, dtype = k.shape[0], self.cfg.kv_heads, self.cfg.head_dim, self.device, k.dtype
        q_heads, rq, ro = 0, None, None
        if q is not None:
            q_heads = _three("q", q)[1]
            if q_out is None:
                q_out = _new_like(q, cuda_stream, dev)
            rq, ro = _rows("q", q, n, q_heads, D, dev, dtype), _rows("q_out", q_out, n, q_heads, D, dev, dtype)
        t, rk, rv = self._table(table), _rows("k", k, n, heads, D, dev, dtype), _rows("v", v, n, heads, D, dev, dtype)
        at = ctypes.addressof
        _check("lacache_kv_append", self._lib.lacache_kv_append(
            self.h, self._layer(layer), at(t), n, _index("seq", seq, n, dev), _index("pos", pos, n, dev),
            None if rope is None else at(rope.plan), None if rope_pos is None else _index("rope_pos", rope_pos, n, dev),
            _dtype(k), at(rk), at(rv), q_heads, None if rq is None else at(rq), None if ro is None else at(ro),
            _current_stream(cuda_stream, dev)))
        return q_out

    def read(self, seq, pos, table, layer: int = 0, dtype=None, k_out=None, v_out=None, cuda_stream=None):
        """The cached rows (k, v) of n tokens, into ``k_out`` and ``v_out`` or new tensors of ``dtype`` (bf16)."""
        n, heads, D, dev = seq.shape[0], self.cfg.kv_heads, self.cfg.head_dim, self.device
        if k_out is None and v_out is None:
            import torch
            with _results_on(cuda_stream, dev):
                k_out = torch.empty(n, heads, D, dtype=torch.bfloat16 if dtype is None else dtype, device=f"cuda:{dev}")
                v_out = torch.empty_like(k_out)
        some = k_out if k_out is not None else v_out
        lacache_kv_read(self.h, self._layer(layer), self._table(table), n, _index("seq", seq, n, dev), _index("pos", pos, n, dev),
                        _dtype(some), None if k_out is None else _rows("k_out", k_out, n, heads, D, dev, some.dtype),
                        None if v_out is None else _rows("v_out", v_out, n, heads, D, dev, some.dtype),
                        _current_stream(cuda_stream, dev))
        return k_out, v_out

    def attend(self, q, table, lengths, new_tokens: int = 1, layer: int = 0, starts=None, window: int = 0,
               scale: float | None = None, out=None, lse=None, cuda_stream=None):
        """Attention of the last ``new_tokens`` tokens of each sequence: q [sequences * new_tokens x q_heads x head_dim],
        ``lengths`` (int32) with the new tokens counted. Returns ``out``; ``lse`` (fp32 [tokens x q_heads]) is filled if
        given. ``scale`` is 1 / sqrt(head_dim) if None. ``out`` does not overlap ``q``."""
        heads, D, dev, dtype = _three("q", q)[1], self.cfg.head_dim, self.device, q.dtype
        t = self._table(table)
        n = t.seqs * new_tokens
        if out is None:
            out = _new_like(q, cuda_stream, dev)
        if lse is not None:
            import torch
            if lse.dtype != torch.float32 or lse.shape != (n, heads) or not lse.is_contiguous() or lse.get_device() != dev:
                raise ValueError(f"lse is a dense fp32 [{n} x {heads}] tensor on cuda:{dev}")
        if not 0 <= window < 1 << 31:
            if window < 0:
                raise ValueError(f"window is a number of positions, or 0 for none, not {window}")
            window = 0   # no position lies further back
        a = lacache_attention(new_tokens, heads, window, _dtype(q), D ** -0.5 if scale is None else scale,
                              _index("lengths", lengths, t.seqs, dev),
                              None if starts is None else _index("starts", starts, t.seqs, dev),
                              _rows("q", q, n, heads, D, dev, dtype), _rows("out", out, n, heads, D, dev, dtype),
                              None if lse is None else lse.data_ptr())
        _check("lacache_kv_attend", self._lib.lacache_kv_attend(
            self.h, self._layer(layer), ctypes.addressof(t), ctypes.addressof(a), _current_stream(cuda_stream, dev)))
        return out

    def sync(self) -> None:
        lacache_kv_sync(self.h)
