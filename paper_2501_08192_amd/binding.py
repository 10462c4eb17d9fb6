"""ctypes binding of libpreserve_mi355x.so: the same entry points as include/preserve.h, include/preserve_aux.h and
include/preserve_ops.h.

Argument marshalling only -- every step of the decode path runs inside the library's HIP kernels.
There is no fallback: if the built library is missing, loading raises.  Device buffers are torch
tensors (or raw integer device addresses); streams are torch.cuda.Stream objects or raw handles.
"""
import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpreserve_mi355x.so")

PSV_OK, PSV_ERR_INVALID_ARG, PSV_ERR_BAD_STATE, PSV_ERR_UNSUPPORTED, PSV_ERR_HIP, PSV_ERR_NOMEM = 0, -1, -2, -3, -4, -5
PSV_ERR_TIMEOUT = -6
PSV_TARGET_WEIGHTS, PSV_TARGET_KV = 1, 2
PSV_OP_QKV, PSV_OP_ATTN, PSV_OP_O, PSV_OP_GATE, PSV_OP_UP, PSV_OP_DOWN = range(6)
OP_NAMES = ["qkv", "attn", "o", "gate", "up", "down"]
PSV_FMT_BF16, PSV_FMT_INT8 = 0, 1
FORMATS = {"bf16": PSV_FMT_BF16, "int8": PSV_FMT_INT8}
PSV_KV_HEAD_MAJOR, PSV_KV_TOKEN_MAJOR = 0, 1
KV_LAYOUTS = {"head": PSV_KV_HEAD_MAJOR, "token": PSV_KV_TOKEN_MAJOR}
PSV_W_ROW_MAJOR, PSV_W_TILED = 0, 1
WEIGHT_LAYOUTS = {"row": PSV_W_ROW_MAJOR, "tiled": PSV_W_TILED}
PSV_KV_UNIT_BYTES_BF16, PSV_KV_UNIT_BYTES_INT8 = 4096, 2112
PSV_STATIC_SCRATCH_BYTES = 16 << 20
PSV_F32, PSV_BF16, PSV_F16 = 0, 1, 2
PSV_ROPE_MAX_DIMS = 256
ROPE_PAIRINGS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "turns": 2, "channel": 3}
PSV_SLOTS_MAX_BATCH = 4096
PSV_LOGPROBS_MAX_TOP, PSV_LOGPROBS_MAX_GIVEN, PSV_LOGPROBS_MAX_RECORDS = 32, 32, 256
PSV_DBG_H1, PSV_DBG_QKV, PSV_DBG_ATTN, PSV_DBG_Y, PSV_DBG_H2, PSV_DBG_M = range(6)

EXPORTS = [
    "psv_strerror", "psv_validate_desc", "psv_workspace_bytes", "psv_plan_chain", "psv_create", "psv_destroy",
    "psv_set_layer_weights", "psv_set_kv", "psv_set_comm_windows", "psv_set_policy", "psv_plan",
    "psv_set_graph_mode", "psv_decode_step", "psv_sync", "psv_get_stats", "psv_tune_attention", "psv_set_attention_chunk", "psv_get_attention_chunk",
    "psv_check_overlap",
    "psv_set_profile_op",
    "psv_get_profile", "psv_prefetch_region", "psv_spin", "psv_copy_bytes", "psv_debug_read",
    "psv_debug_force_wait_timeout", "psv_decode_step_static", "psv_set_fused_kernels", "psv_debug_last_step_path", "psv_debug_last_step_prelaunches", "psv_debug_last_step_read_once", "psv_tile_weights",
]

# the operators around the decode step (include/preserve_ops.h)
OPERATOR_EXPORTS = [
    "psv_rope_plan", "psv_set_rope", "psv_rotate", "psv_cache_slots", "psv_cache_append", "psv_cache_gather", "psv_logprobs_records",
    "psv_logprobs_bytes", "psv_logprobs_part", "psv_logprobs_join", "psv_logprobs",
]


class psv_model_desc(C.Structure):
    _fields_ = [("n_layers", C.c_uint32), ("hidden", C.c_uint32), ("n_q_heads", C.c_uint32),
                ("n_kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("ffn", C.c_uint32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("max_batch", C.c_uint32),
                ("max_seq", C.c_uint32), ("weight_format", C.c_uint32), ("kv_format", C.c_uint32),
                ("kv_layout", C.c_uint32), ("weight_layout", C.c_uint32)]


class psv_layer_weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_qkv", "w_o", "w_gate", "w_up", "w_down", "g_attn", "g_mlp",
                                          "s_qkv", "s_o", "s_gate", "s_up", "s_down")]


class psv_kv_desc(C.Structure):
    _fields_ = [("k_pools", C.POINTER(C.c_void_p)), ("v_pools", C.POINTER(C.c_void_p)),
                ("page_table", C.c_void_p), ("max_blocks", C.c_uint32), ("num_pool_blocks", C.c_uint32),
                ("seq_lens", C.c_void_p)]


class psv_prefetch_policy(C.Structure):
    _fields_ = [("mode", C.c_uint32), ("targets", C.c_uint32), ("budget_bytes", C.c_uint64),
                ("chunk_bytes", C.c_uint64), ("cu_budget", C.c_uint32), ("partial", C.c_uint32),
                ("join", C.c_uint32), ("prelaunch", C.c_uint32)]


class psv_plan_entry(C.Structure):
    _fields_ = [("layer", C.c_uint32), ("window", C.c_uint32), ("target_layer", C.c_uint32),
                ("target_op", C.c_uint32), ("mem_size", C.c_uint64), ("bytes", C.c_uint64)]


class psv_stats(C.Structure):
    _fields_ = [("weight_bytes_per_layer", C.c_uint64), ("kv_bytes_per_layer", C.c_uint64),
                ("planned_prefetch_bytes", C.c_uint64), ("workspace_bytes", C.c_uint64),
                ("kernels_per_layer", C.c_uint32), ("prefetch_launches", C.c_uint32),
                ("steps", C.c_uint32), ("reserved", C.c_uint32)]


class psv_rope_desc(C.Structure):
    _fields_ = [("dims", C.c_uint32), ("pairing", C.c_uint32), ("scaling", C.c_uint32), ("reserved", C.c_uint32),
                ("magnitude", C.c_double),
                ("theta", C.c_double), ("factor", C.c_double), ("low_turns", C.c_double), ("high_turns", C.c_double),
                ("trained_context", C.c_double)]


class psv_rope(C.Structure):
    _fields_ = [("dims", C.c_uint32), ("pairing", C.c_uint32), ("magnitude", C.c_double),
                ("freq", C.c_double * (PSV_ROPE_MAX_DIMS // 2))]


class psv_rotate_args(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("positions", C.c_void_p), ("rows", C.c_uint32), ("heads", C.c_uint32),
                ("head_dim", C.c_uint32), ("dtype", C.c_uint32), ("transpose", C.c_uint32), ("reserved", C.c_uint32),
                ("x_row", C.c_int64), ("x_head", C.c_int64), ("y_row", C.c_int64), ("y_head", C.c_int64)]


class psv_slots_args(C.Structure):
    _fields_ = [("lens", C.c_void_p), ("new_lens", C.c_void_p), ("block_table", C.c_void_p), ("free_blocks", C.c_void_p),
                ("free_range", C.c_void_p), ("free_capacity", C.c_uint32), ("batch", C.c_uint32), ("max_blocks", C.c_uint32),
                ("num_pool_blocks", C.c_uint32), ("rows", C.c_uint32), ("reserved", C.c_uint32), ("seq_lens", C.c_void_p),
                ("row_starts", C.c_void_p), ("slots", C.c_void_p), ("positions", C.c_void_p), ("requests", C.c_void_p),
                ("free_range_out", C.c_void_p), ("refused", C.c_void_p)]


class psv_cache(C.Structure):
    device = None      # of the pools, where they were given as tensors
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("n_kv_heads", C.c_uint32), ("kv_format", C.c_uint32),
                ("kv_layout", C.c_uint32), ("num_pool_blocks", C.c_uint32)]


class psv_append_args(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_out", C.c_void_p), ("positions", C.c_void_p),
                ("slots", C.c_void_p), ("rows", C.c_uint32), ("n_q_heads", C.c_uint32), ("dtype", C.c_uint32),
                ("reserved", C.c_uint32), ("q_row", C.c_int64), ("k_row", C.c_int64), ("v_row", C.c_int64),
                ("q_out_row", C.c_int64)]


class psv_gather_args(C.Structure):
    _fields_ = [("slots", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("rows", C.c_uint32), ("dtype", C.c_uint32),
                ("k_row", C.c_int64), ("v_row", C.c_int64)]


class psv_logprobs_args(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("tokens", C.c_void_p), ("rows", C.c_uint32), ("columns", C.c_uint32),
                ("first_token", C.c_uint32), ("vocab", C.c_uint32), ("dtype", C.c_uint32), ("given", C.c_uint32),
                ("top", C.c_uint32), ("scale", C.c_float), ("records", C.c_uint32), ("reserved", C.c_uint32), ("row", C.c_int64)]


class psv_logprobs_out(C.Structure):
    _fields_ = [("logprobs", C.c_void_p), ("entropy", C.c_void_p), ("top_logprobs", C.c_void_p), ("top_ids", C.c_void_p)]


class PsvError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, strerror(status), status))


_lib = None


def lib():
    """Loads the built library; raises if it has not been built (there is no other code path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libpreserve_mi355x.so is not built: run `python -c 'import __graft_entry__ as g; "
                              "g.build()'` or `python paper_2501_08192_amd/build.py`")
        L = C.CDLL(LIB_PATH)
        vp, u32, u64, sz = C.c_void_p, C.c_uint32, C.c_uint64, C.c_size_t
        sig = {
            "psv_strerror": (C.c_char_p, [C.c_int32]),
            "psv_validate_desc": (C.c_int32, [C.POINTER(psv_model_desc)]),
            "psv_workspace_bytes": (sz, [C.POINTER(psv_model_desc)]),
            "psv_plan_chain": (C.c_int32, [C.POINTER(psv_model_desc), u32, u32, C.POINTER(psv_prefetch_policy),
                                           C.POINTER(psv_plan_entry), sz, C.POINTER(sz)]),
            "psv_create": (C.c_int32, [C.POINTER(psv_model_desc), vp, vp, C.POINTER(vp)]),
            "psv_destroy": (C.c_int32, [vp]),
            "psv_set_layer_weights": (C.c_int32, [vp, u32, C.POINTER(psv_layer_weights)]),
            "psv_set_kv": (C.c_int32, [vp, C.POINTER(psv_kv_desc)]),
            "psv_set_comm_windows": (C.c_int32, [vp, C.c_float, C.c_float]),
            "psv_set_policy": (C.c_int32, [vp, C.POINTER(psv_prefetch_policy), u32, u32]),
            "psv_plan": (C.c_int32, [vp, C.POINTER(psv_plan_entry), sz, C.POINTER(sz)]),
            "psv_set_graph_mode": (C.c_int32, [vp, u32]),
            "psv_decode_step": (C.c_int32, [vp, vp, vp, u32, u32, u32]),
            "psv_sync": (C.c_int32, [vp]),
            "psv_get_stats": (C.c_int32, [vp, C.POINTER(psv_stats)]),
            "psv_tune_attention": (C.c_int32, [vp, vp, vp, u32, C.POINTER(u32)]),
            "psv_set_attention_chunk": (C.c_int32, [vp, u32]),
            "psv_get_attention_chunk": (C.c_int32, [vp, C.POINTER(u32)]),
            "psv_check_overlap": (C.c_int32, [vp, C.POINTER(C.c_int32)]),
            "psv_set_profile_op": (C.c_int32, [vp, C.c_int32]),
            "psv_get_profile": (C.c_int32, [vp, C.POINTER(C.c_double), C.POINTER(u64)]),
            "psv_prefetch_region": (C.c_int32, [vp, u64, u32, vp]),
            "psv_spin": (C.c_int32, [C.c_float, vp]),
            "psv_copy_bytes": (C.c_int32, [vp, vp, u64, vp]),
            "psv_debug_read": (C.c_int32, [vp, u32, vp, sz]),
            "psv_debug_force_wait_timeout": (C.c_int32, [vp, u32]),
            "psv_debug_last_step_path": (C.c_int32, [vp, C.POINTER(u32)]),
            "psv_debug_last_step_prelaunches": (C.c_int32, [vp, C.POINTER(u32)]),
            "psv_debug_last_step_read_once": (C.c_int32, [vp, C.POINTER(u32)]),
            "psv_tile_weights": (C.c_int32, [vp, vp, u32, u32, u32, vp]),
            "psv_set_fused_kernels": (C.c_int32, [vp, u32]),
            "psv_decode_step_static": (C.c_int32, [C.POINTER(psv_model_desc), C.POINTER(psv_layer_weights),
                                                   C.POINTER(psv_kv_desc), vp, vp, u32, u32, u32, vp]),
            "psv_rope_plan": (C.c_int32, [C.POINTER(psv_rope_desc), C.POINTER(psv_rope)]),
            "psv_set_rope": (C.c_int32, [vp, C.POINTER(psv_rope)]),
            "psv_rotate": (C.c_int32, [C.POINTER(psv_rotate_args), C.POINTER(psv_rope), vp]),
            "psv_cache_slots": (C.c_int32, [C.POINTER(psv_slots_args), vp]),
            "psv_cache_append": (C.c_int32, [C.POINTER(psv_append_args), C.POINTER(psv_cache), C.POINTER(psv_rope), vp]),
            "psv_cache_gather": (C.c_int32, [C.POINTER(psv_gather_args), C.POINTER(psv_cache), vp]),
            "psv_logprobs_records": (u32, [u32, u32]),
            "psv_logprobs_bytes": (sz, [u32, u32, u32, u32]),
            "psv_logprobs_part": (C.c_int32, [C.POINTER(psv_logprobs_args), vp, vp]),
            "psv_logprobs_join": (C.c_int32, [C.POINTER(psv_logprobs_args), vp, u32, C.POINTER(psv_logprobs_out), vp]),
            "psv_logprobs": (C.c_int32, [C.POINTER(psv_logprobs_args), C.POINTER(psv_logprobs_out), vp, sz, vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status, where):
    if status != PSV_OK:
        raise PsvError(status, where)


def _dev_ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(s):
    if s is None or isinstance(s, int):
        return s
    return s.cuda_stream


def strerror(status):
    return lib().psv_strerror(int(status)).decode()


def model_desc(n_layers, hidden, n_q_heads, n_kv_heads, ffn, max_batch, max_seq, head_dim=128, rms_eps=1e-5,
               rope_theta=500000.0, weight_format="bf16", kv_format="bf16", kv_layout="head", weight_layout="row"):
    return psv_model_desc(n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, rms_eps, rope_theta, max_batch,
                          max_seq, FORMATS[weight_format], FORMATS[kv_format], KV_LAYOUTS[kv_layout], WEIGHT_LAYOUTS[weight_layout])


def prefetch_policy(mode=0, targets=PSV_TARGET_WEIGHTS | PSV_TARGET_KV, budget_bytes=0, chunk_bytes=0, cu_budget=0,
                    partial=0, join=0, prelaunch=0):
    return psv_prefetch_policy(mode, targets, budget_bytes, chunk_bytes, cu_budget, partial, join, prelaunch)


def psv_validate_desc(desc):
    return int(lib().psv_validate_desc(C.byref(desc)))


def psv_workspace_bytes(desc):
    return int(lib().psv_workspace_bytes(C.byref(desc)))


def _entries(arr, n):
    return [dict(layer=e.layer, window=e.window, target_layer=e.target_layer, target_op=e.target_op,
                 mem_size=e.mem_size, bytes=e.bytes) for e in arr[:n]]


def psv_plan_chain(desc, batch, context, policy):
    n = C.c_size_t(0)
    _check(lib().psv_plan_chain(C.byref(desc), batch, context, C.byref(policy), None, 0, C.byref(n)), "psv_plan_chain")
    arr = (psv_plan_entry * max(1, n.value))()
    _check(lib().psv_plan_chain(C.byref(desc), batch, context, C.byref(policy), arr, n.value, C.byref(n)), "psv_plan_chain")
    return _entries(arr, n.value)


def psv_create(desc, stream_main, stream_side):
    out = C.c_void_p()
    _check(lib().psv_create(C.byref(desc), _stream(stream_main), _stream(stream_side), C.byref(out)), "psv_create")
    return out


def psv_destroy(ctx):
    _check(lib().psv_destroy(ctx), "psv_destroy")


def psv_set_layer_weights(ctx, layer, weights):
    """weights: dict name -> device tensor: w_qkv, w_o, w_gate, w_up, w_down (bf16, or int8 codes), g_attn, g_mlp
    (bf16) and, for int8 weights, the fp32 per-row scales s_qkv, s_o, s_gate, s_up, s_down."""
    w = psv_layer_weights(*[_dev_ptr(weights.get(n)) for n, _ in psv_layer_weights._fields_])
    _check(lib().psv_set_layer_weights(ctx, layer, C.byref(w)), "psv_set_layer_weights")


def psv_set_kv(ctx, k_pools, v_pools, page_table, max_blocks, num_pool_blocks, seq_lens):
    n = len(k_pools)
    ka = (C.c_void_p * n)(*[_dev_ptr(t) for t in k_pools])
    va = (C.c_void_p * n)(*[_dev_ptr(t) for t in v_pools])
    kv = psv_kv_desc(ka, va, _dev_ptr(page_table), max_blocks, num_pool_blocks, _dev_ptr(seq_lens))
    _check(lib().psv_set_kv(ctx, C.byref(kv)), "psv_set_kv")


def psv_set_comm_windows(ctx, us_after_attn, us_after_mlp):
    _check(lib().psv_set_comm_windows(ctx, us_after_attn, us_after_mlp), "psv_set_comm_windows")


def psv_set_policy(ctx, policy, batch, context):
    _check(lib().psv_set_policy(ctx, C.byref(policy), batch, context), "psv_set_policy")


def psv_plan(ctx):
    n = C.c_size_t(0)
    _check(lib().psv_plan(ctx, None, 0, C.byref(n)), "psv_plan")
    arr = (psv_plan_entry * max(1, n.value))()
    _check(lib().psv_plan(ctx, arr, n.value, C.byref(n)), "psv_plan")
    return _entries(arr, n.value)


def psv_set_graph_mode(ctx, use_graph):
    _check(lib().psv_set_graph_mode(ctx, 1 if use_graph else 0), "psv_set_graph_mode")


def psv_decode_step(ctx, x_in, x_out, batch, layer_begin, layer_end):
    _check(lib().psv_decode_step(ctx, _dev_ptr(x_in), _dev_ptr(x_out), batch, layer_begin, layer_end), "psv_decode_step")


def psv_decode_step_static(desc, layers, k_pools, v_pools, page_table, max_blocks, num_pool_blocks, seq_lens, x_in, x_out,
                           batch, layer_begin, layer_end, stream):
    """layers: list (one entry per layer of desc; None where a layer is outside the range) of weight dicts as for
    psv_set_layer_weights; k_pools / v_pools: lists of device tensors, one per layer."""
    n = len(layers)
    arr = (psv_layer_weights * n)()
    for i, w in enumerate(layers):
        if w is not None:
            arr[i] = psv_layer_weights(*[_dev_ptr(w.get(f)) for f, _ in psv_layer_weights._fields_])
    ka = (C.c_void_p * n)(*[_dev_ptr(t) for t in k_pools])
    va = (C.c_void_p * n)(*[_dev_ptr(t) for t in v_pools])
    kv = psv_kv_desc(ka, va, _dev_ptr(page_table), max_blocks, num_pool_blocks, _dev_ptr(seq_lens))
    _check(lib().psv_decode_step_static(C.byref(desc), arr, C.byref(kv), _dev_ptr(x_in), _dev_ptr(x_out), batch,
                                        layer_begin, layer_end, _stream(stream)), "psv_decode_step_static")


def psv_sync(ctx):
    _check(lib().psv_sync(ctx), "psv_sync")


def psv_get_stats(ctx):
    s = psv_stats()
    _check(lib().psv_get_stats(ctx, C.byref(s)), "psv_get_stats")
    return {n: getattr(s, n) for n, _ in psv_stats._fields_ if n != "reserved"}


def psv_tune_attention(ctx, x_in, x_out, batch):
    out = C.c_uint32(0)
    _check(lib().psv_tune_attention(ctx, _dev_ptr(x_in), _dev_ptr(x_out), batch, C.byref(out)), "psv_tune_attention")
    return int(out.value)


def psv_set_attention_chunk(ctx, chunk_tokens):
    _check(lib().psv_set_attention_chunk(ctx, int(chunk_tokens)), "psv_set_attention_chunk")


def psv_get_attention_chunk(ctx):
    out = C.c_uint32(0)
    _check(lib().psv_get_attention_chunk(ctx, C.byref(out)), "psv_get_attention_chunk")
    return int(out.value)


def psv_check_overlap(ctx):
    out = C.c_int32(0)
    _check(lib().psv_check_overlap(ctx, C.byref(out)), "psv_check_overlap")
    return bool(out.value)


def psv_set_profile_op(ctx, op):
    _check(lib().psv_set_profile_op(ctx, op), "psv_set_profile_op")


def psv_get_profile(ctx):
    ms, n = C.c_double(0), C.c_uint64(0)
    _check(lib().psv_get_profile(ctx, C.byref(ms), C.byref(n)), "psv_get_profile")
    return ms.value, n.value


def psv_prefetch_region(ptr, nbytes, workgroups, stream):
    _check(lib().psv_prefetch_region(_dev_ptr(ptr), nbytes, workgroups, _stream(stream)), "psv_prefetch_region")


def psv_spin(us, stream):
    _check(lib().psv_spin(us, _stream(stream)), "psv_spin")


def psv_copy_bytes(dst, src, nbytes, stream):
    _check(lib().psv_copy_bytes(_dev_ptr(dst), _dev_ptr(src), nbytes, _stream(stream)), "psv_copy_bytes")


def psv_debug_read(ctx, which, host_array):
    """host_array: a contiguous numpy array that receives the buffer."""
    _check(lib().psv_debug_read(ctx, which, host_array.ctypes.data_as(C.c_void_p), host_array.nbytes), "psv_debug_read")
    return host_array


def psv_set_fused_kernels(ctx, on):
    """on: 0 / False = one kernel per operator, 1 / True = one per block, 2 = the whole step as one kernel."""
    _check(lib().psv_set_fused_kernels(ctx, int(on)), "psv_set_fused_kernels")


def psv_tile_weights(dst, src, rows, cols, weight_format, stream):
    """dst, src: device tensors of rows * cols elements; weight_format "bf16" or "int8"."""
    _check(lib().psv_tile_weights(_dev_ptr(dst), _dev_ptr(src), int(rows), int(cols), FORMATS[weight_format], _stream(stream)),
           "psv_tile_weights")


def psv_debug_last_step_path(ctx):
    out = C.c_uint32(0)
    _check(lib().psv_debug_last_step_path(ctx, C.byref(out)), "psv_debug_last_step_path")
    return int(out.value)


def psv_debug_last_step_prelaunches(ctx):
    out = C.c_uint32(0)
    _check(lib().psv_debug_last_step_prelaunches(ctx, C.byref(out)), "psv_debug_last_step_prelaunches")
    return int(out.value)


def psv_debug_last_step_read_once(ctx):
    """(weights, keys and values): read non-temporally in the last step?"""
    out = C.c_uint32(0)
    _check(lib().psv_debug_last_step_read_once(ctx, C.byref(out)), "psv_debug_last_step_read_once")
    return bool(out.value & 1), bool(out.value & 2)


def psv_debug_force_wait_timeout(ctx, on):
    _check(lib().psv_debug_force_wait_timeout(ctx, 1 if on else 0), "psv_debug_force_wait_timeout")


# ---- operators around the decode step (include/preserve_ops.h) -----------------------------------------------------------


_TYPES = {}      # a tensor's dtype -> its name; filled as types are seen


def _type(t):
    name = _TYPES.get(t.dtype)
    if name is None:
        name = _TYPES[t.dtype] = str(t.dtype).replace("torch.", "")
    return name


_ROW_TYPES = {"float32": PSV_F32, "bfloat16": PSV_BF16, "float16": PSV_F16}
_ROW_CODES = {}  # ... -> its code as rows' element type


def _dtype(name, t):
    code = _ROW_CODES.get(t.dtype)
    if code is None:
        code = _ROW_TYPES.get(_type(t))
        if code is None:
            raise ValueError("%s: float32, bfloat16 or float16 is wanted, got %s" % (name, t.dtype))
        _ROW_CODES[t.dtype] = code
    return code


def _device(stream, t):
    """The GPU that a call's tensors lie on: its stream's, or, of a stream that is only a handle, that of its first tensor."""
    at = getattr(stream, "device_index", None)
    return t.get_device() if at is None else at


def _elsewhere(name, t):
    raise ValueError("%s: a tensor on the stream's GPU is wanted, got one on %s" % (name, t.device))


def _place(name, t, at):
    """The address of a tensor on GPU `at`: kernels follow it."""
    if t.get_device() != at or at < 0:
        _elsewhere(name, t)
    return t.data_ptr()


def _rows(name, t, at):
    """(dtype code, row stride, shape, address) of rows [rows, heads, channels] on GPU `at` whose heads and channels are adjacent."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[2] != 128 or stride[2] != 1 or (shape[1] > 1 and stride[1] != 128):
        raise ValueError("%s: rows of [heads][128] adjacent elements are wanted, got shape %s, strides %s" % (name, tuple(shape), stride))
    if t.get_device() != at or at < 0:
        _elsewhere(name, t)
    code = _ROW_CODES.get(t.dtype)
    return _dtype(name, t) if code is None else code, stride[0], shape, t.data_ptr()


def _want(name, t, at, dtype, *shape):
    """The address of a contiguous tensor of a type and shape on GPU `at`."""
    if (_TYPES.get(t.dtype) or _type(t)) != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: contiguous %s %s is wanted, got %s %s" % (name, dtype, list(shape), t.dtype, list(t.shape)))
    if t.get_device() != at or at < 0:
        _elsewhere(name, t)
    return t.data_ptr()


def _bytes_at(name, t, at, n):
    """The address of a contiguous tensor of `n` bytes or more; nothing for none."""
    if t is None and n == 0:
        return None
    if not t.is_contiguous() or t.numel() * t.element_size() < n:
        raise ValueError("%s: a contiguous tensor of at least %d bytes is wanted, got %s of %s" % (name, n, list(t.shape), t.dtype))
    return _place(name, t, at)


def psv_rope_plan(dims=128, pairing="half", theta=500000.0, scaling="plain", factor=1.0, low_turns=1.0, high_turns=4.0,
                  trained_context=8192.0, magnitude=1.0):
    """Frequencies for psv_rotate, psv_cache_append and psv_set_rope; pairing and scaling: keys of ROPE_PAIRINGS and ROPE_SCALINGS."""
    desc = psv_rope_desc(dims, ROPE_PAIRINGS[pairing], ROPE_SCALINGS[scaling], 0, magnitude, theta, factor, low_turns, high_turns, trained_context)
    out = psv_rope()
    _check(lib().psv_rope_plan(C.byref(desc), C.byref(out)), "psv_rope_plan")
    return out


def psv_set_rope(ctx, rope):
    _check(lib().psv_set_rope(ctx, None if rope is None else C.byref(rope)), "psv_set_rope")


def psv_rotate(x, y, positions, rope, stream, transpose=False):
    """x, y: [rows, heads, channels] of one type, any strides with adjacent channels; positions: int32 [rows]."""
    shape, xs, ys = x.shape, x.stride(), y.stride()
    if len(shape) != 3 or y.shape != shape or y.dtype != x.dtype or (shape[2] > 1 and (xs[2] != 1 or ys[2] != 1)):
        raise ValueError("psv_rotate: x and y of one shape [rows, heads, channels] and type with adjacent channels are wanted")
    at = _device(stream, x)
    a = psv_rotate_args(_place("x", x, at), _place("y", y, at), _want("positions", positions, at, "int32", shape[0]), shape[0], shape[1], shape[2], _dtype("x", x),
                        1 if transpose else 0, 0, xs[0], xs[1], ys[0], ys[1])
    _check(lib().psv_rotate(C.byref(a), C.byref(rope), _stream(stream)), "psv_rotate")


def psv_cache_slots(lens, new_lens, block_table, free_blocks, free_range, num_pool_blocks, seq_lens, row_starts, slots, positions,
                    requests, free_range_out, refused, stream, max_blocks=None):
    """Tensors as in psv_slots_args (int32; slots int64); block_table, free_blocks, free_range, free_range_out None and max_blocks given
    for a contiguous cache."""
    n, rows = lens.shape[0], slots.shape[0]
    table = block_table is not None
    mb, n_free = (block_table.shape[-1], free_blocks.shape[0]) if table else (int(max_blocks), 0)
    at = _device(stream, lens)
    a = psv_slots_args(_want("lens", lens, at, "int32", n), _want("new_lens", new_lens, at, "int32", n),
                       _want("block_table", block_table, at, "int32", n, mb) if table else None,
                       _want("free_blocks", free_blocks, at, "int32", n_free) if table else None,
                       _want("free_range", free_range, at, "int32", 2) if table else None, n_free, n, mb, num_pool_blocks, rows, 0,
                       _want("seq_lens", seq_lens, at, "int32", n), _want("row_starts", row_starts, at, "int32", n + 1),
                       _want("slots", slots, at, "int64", rows), _want("positions", positions, at, "int32", rows),
                       _want("requests", requests, at, "int32", rows),
                       _want("free_range_out", free_range_out, at, "int32", 2) if table else None, _want("refused", refused, at, "int32", 1))
    _check(lib().psv_cache_slots(C.byref(a), _stream(stream)), "psv_cache_slots")


def kv_cache(k_pool, v_pool, n_kv_heads, kv_format, kv_layout, num_pool_blocks):
    """One layer's pools, tensors on one GPU or addresses; kv_format, kv_layout: keys of FORMATS and KV_LAYOUTS."""
    if k_pool is None or v_pool is None or isinstance(k_pool, int) or isinstance(v_pool, int):
        for t in (k_pool, v_pool):
            if t is not None and not isinstance(t, int):
                _place("pool", t, t.get_device())
        return psv_cache(_dev_ptr(k_pool), _dev_ptr(v_pool), n_kv_heads, FORMATS[kv_format], KV_LAYOUTS[kv_layout], num_pool_blocks)
    at = k_pool.get_device()
    cache = psv_cache(_place("k_pool", k_pool, at), _place("v_pool", v_pool, at), n_kv_heads, FORMATS[kv_format], KV_LAYOUTS[kv_layout], num_pool_blocks)
    cache.device = at
    return cache


def _other_gpu(cache, at):
    raise ValueError("cache: its pools lie on GPU %d, the call's tensors on GPU %d" % (cache.device, at))


def psv_cache_append(q, k, v, q_out, positions, slots, cache, rope, stream):
    """q, q_out [rows, q heads, 128], or None; k, v [rows, kv heads, 128]; positions int32 [rows] (None without rope); slots int64 [rows]."""
    at = _device(stream, k)
    dt, k_row, shape, k_at = _rows("k", k, at)
    dv, v_row, v_shape, v_at = _rows("v", v, at)
    if dv != dt or v_shape != shape or shape[1] != cache.n_kv_heads:
        raise ValueError("psv_cache_append: k and v of one type with the cache's %d heads are wanted" % cache.n_kv_heads)
    rows, nq, q_row, q_out_row, q_at, q_out_at = shape[0], 0, 0, 0, None, None
    if q is not None:
        dq, q_row, q_shape, q_at = _rows("q", q, at)
        do, q_out_row, q_out_shape, q_out_at = _rows("q_out", q_out, at)
        if dq != dt or do != dt or q_out_shape != q_shape or q_shape[0] != rows:
            raise ValueError("psv_cache_append: q and q_out of k's type and rows are wanted")
        nq = q_shape[1]
    if cache.device != at and cache.device is not None:
        _other_gpu(cache, at)
    a = psv_append_args(q_at, k_at, v_at, q_out_at, None if positions is None else _want("positions", positions, at, "int32", rows),
                        _want("slots", slots, at, "int64", rows), rows, nq, dt, 0, q_row, k_row, v_row, q_out_row)
    _check(lib().psv_cache_append(C.byref(a), C.byref(cache), None if rope is None else C.byref(rope), _stream(stream)), "psv_cache_append")


def psv_cache_gather(slots, k, v, cache, stream):
    """slots int64 [rows]; k, v [rows, kv heads, 128] of one type."""
    rows = slots.shape[0]
    at = _device(stream, k)
    dt, k_row, shape, k_at = _rows("k", k, at)
    dv, v_row, v_shape, v_at = _rows("v", v, at)
    if dv != dt or v_shape != shape or shape[0] != rows or shape[1] != cache.n_kv_heads:
        raise ValueError("psv_cache_gather: k and v of one type with %d rows of the cache's %d heads are wanted" % (rows, cache.n_kv_heads))
    if cache.device != at and cache.device is not None:
        _other_gpu(cache, at)
    a = psv_gather_args(_want("slots", slots, at, "int64", rows), k_at, v_at, rows, dt, k_row, v_row)
    _check(lib().psv_cache_gather(C.byref(a), C.byref(cache), _stream(stream)), "psv_cache_gather")


def psv_logprobs_records(rows, columns):
    return int(lib().psv_logprobs_records(rows, columns))


def psv_logprobs_bytes(rows, records, given, top):
    return int(lib().psv_logprobs_bytes(rows, records, given, top))


def _logprobs_args(at, rows, logits, tokens, scale, top, first_token, vocab, records):
    given = 0 if tokens is None else tokens.shape[1]
    columns, row, dt, where = 0, 0, PSV_F32, None
    if logits is not None:
        shape, stride = logits.shape, logits.stride()
        if len(shape) != 2 or shape[0] != rows or (shape[1] > 1 and stride[1] != 1):
            raise ValueError("logits: [rows, columns] with adjacent columns are wanted")
        columns, row, dt, where = shape[1], stride[0], _dtype("logits", logits), _place("logits", logits, at)
    return psv_logprobs_args(where, None if given == 0 else _want("tokens", tokens, at, "int32", rows, given), rows, columns, first_token,
                             columns if vocab is None else vocab, dt, given, top, scale, records, 0, row)


def _logprobs_out(at, rows, given, logprobs, entropy, top_logprobs, top_ids):
    if (top_ids is None) != (top_logprobs is None):
        raise ValueError("top_logprobs, top_ids: both or neither are wanted")
    top = 0 if top_ids is None else top_ids.shape[1]
    return psv_logprobs_out(None if logprobs is None else _want("logprobs", logprobs, at, "float32", rows, given),
                            None if entropy is None else _want("entropy", entropy, at, "float32", rows),
                            None if top == 0 else _want("top_logprobs", top_logprobs, at, "float32", rows, top),
                            None if top == 0 else _want("top_ids", top_ids, at, "int32", rows, top)), top


def psv_logprobs_part(logits, tokens, scale, top, records_out, stream, first_token=0, vocab=None, records=0):
    """logits [rows, columns]: a shard's columns of the vocabulary; tokens int32 [rows, given] or None; records_out: a contiguous tensor of at
    least psv_logprobs_bytes bytes."""
    rows, at = logits.shape[0], _device(stream, logits)
    a = _logprobs_args(at, rows, logits, tokens, scale, top, first_token, vocab, records)
    size = psv_logprobs_bytes(rows, records or psv_logprobs_records(rows, a.columns), a.given, top)
    _check(lib().psv_logprobs_part(C.byref(a), _bytes_at("records_out", records_out, at, size), _stream(stream)), "psv_logprobs_part")


def psv_logprobs_join(rows, tokens, scale, vocab, records, shards, logprobs, entropy, top_logprobs, top_ids, records_in, stream, top=None):
    """records_in: the shards' records of psv_logprobs_part behind one another; top: of the records (top_ids's width by default)."""
    at = _device(stream, records_in)
    out, n = _logprobs_out(at, rows, 0 if tokens is None else tokens.shape[1], logprobs, entropy, top_logprobs, top_ids)
    if top is not None and n not in (0, top):
        raise ValueError("psv_logprobs_join: top_ids is [rows, top]")
    a = _logprobs_args(at, rows, None, tokens, scale, n if top is None else top, 0, vocab, records)
    size = shards * psv_logprobs_bytes(rows, records, a.given, a.top)
    _check(lib().psv_logprobs_join(C.byref(a), _bytes_at("records_in", records_in, at, size), shards, C.byref(out), _stream(stream)), "psv_logprobs_join")


def psv_logprobs(logits, tokens, scale, logprobs, entropy, top_logprobs, top_ids, workspace, stream):
    """logits [rows, vocabulary]; tokens int32 [rows, given] or None; the outputs, any of them None, top_logprobs and top_ids together;
    workspace: a contiguous tensor of at least psv_logprobs_bytes bytes."""
    rows, at = logits.shape[0], _device(stream, logits)
    out, top = _logprobs_out(at, rows, 0 if tokens is None else tokens.shape[1], logprobs, entropy, top_logprobs, top_ids)
    a = _logprobs_args(at, rows, logits, tokens, scale, top, 0, None, 0)
    _check(lib().psv_logprobs(C.byref(a), C.byref(out), _bytes_at("workspace", workspace, at, 0), workspace.numel() * workspace.element_size(),
                              _stream(stream)), "psv_logprobs")
