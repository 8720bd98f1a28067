"""Python binding of libas2d.so, the GB300 (sm_103a) target-side block
verification library (C-ABI: include/as2d.h).

The functions below carry the C names and only marshal arguments: every step
of the verification pass runs in the library's CUDA kernels.  PyTorch is used
by callers for device memory and streams only.  Importing this package fails
loudly if libas2d.so has not been built: there is no fallback path.
"""
import ctypes
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libas2d.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
        "(or python paper_2609_37617_gb300/build.py). There is no CPU fallback.")

_lib = ctypes.CDLL(LIB_PATH)

AS2D_OK = 0
AS2D_ERR_INVALID_ARG = -1
AS2D_ERR_CAPACITY = -2
AS2D_ERR_CUDA = -3
AS2D_ERR_UNSUPPORTED = -4
AS2D_ERR_DEVICE = -5
AS2D_ERR_NO_MEMORY = -6
AS2D_DEVERR_BAD_TOKEN = 1
AS2D_DEVERR_ROLLBACK = 2
AS2D_DEVERR_TIMEOUT = 4
AS2D_DEVERR_CAPACITY = 8
AS2D_DEVERR_BAD_TREE = 16
AS2D_DEVERR_NO_TOKEN = 32
AS2D_DEVERR_NOT_FINITE = 64
AS2D_CBUF_BATCH = 8
CBUF_MODES = {0: "normal", 1: "realign", 2: "alone"}
AS2D_MAX_K = 16
AS2D_MAX_BATCH = 64
AS2D_MAX_TREE = 64
AS2D_TYPE_BF16 = 0
AS2D_TYPE_F32 = 1

EXPORTED = ("as2d_model_load", "as2d_kv_init_prefilled", "as2d_verify_block",
            "as2d_decode_step", "as2d_kv_rollback", "as2d_kv_read_state",
            "as2d_kv_device_state", "as2d_kv_check", "as2d_kv_free",
            "as2d_model_free", "as2d_last_error", "as2d_kv_profile",
            "as2d_kv_profile_read", "as2d_decode_step_static", "as2d_kv_set_wait_limit",
            "as2d_cbuf_create", "as2d_cbuf_publish", "as2d_cbuf_candidates", "as2d_cbuf_after_call",
            "as2d_cbuf_state", "as2d_cbuf_source_of", "as2d_cbuf_free", "as2d_cbuf_held",
            "as2d_verify_from_buffers", "as2d_interval_accounting", "as2d_session_run",
            "as2d_budget_select", "as2d_prefill", "as2d_model_set_sm_budget",
            "as2d_cpu_decoder_create", "as2d_cpu_decoder_step", "as2d_cpu_decoder_logits",
            "as2d_cpu_decoder_reset", "as2d_cpu_decoder_free",
            "as2d_tree_attention_workspace", "as2d_tree_attention", "as2d_attention_weights",
            "as2d_cache_evict_workspace", "as2d_cache_evict", "as2d_token_probs",
            "as2d_accept_sampled", "as2d_verify_tree", "as2d_verify_sampled",
            "as2d_kv_track_weights", "as2d_kv_evict", "as2d_cache_append", "as2d_cache4_append",
            "as2d_cache4_write", "as2d_cache4_read", "as2d_cache4_attention_workspace",
            "as2d_cache4_attention", "as2d_prompt_attention_workspace", "as2d_prompt_attention")
KERNEL_CLASSES = {"qkv": 0, "attention": 1, "o": 2, "gate_up": 3, "down": 4,
                  "lm_head": 5, "other": 6}


class as2d_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rope_theta", ctypes.c_float),
                ("rms_eps", ctypes.c_float)]


class as2d_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "embed", "final_norm", "lm_head", "attn_norm", "w_q", "w_k", "w_v",
        "w_o", "mlp_norm", "w_gate", "w_up", "w_down")]


class as2d_verify_out(ctypes.Structure):
    _fields_ = [("n_accepted", ctypes.c_void_p), ("correction_token", ctypes.c_void_p),
                ("greedy", ctypes.c_void_p), ("logits", ctypes.c_void_p)]


class as2d_source_record(ctypes.Structure):
    _fields_ = [("request", ctypes.c_int32), ("source", ctypes.c_int32),
                ("producer", ctypes.c_int32), ("offset", ctypes.c_int32),
                ("time", ctypes.c_double), ("confidence", ctypes.c_float),
                ("has_confidence", ctypes.c_int32)]


class as2d_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int32) for n in ("n_layers", "batch", "n_kv", "capacity", "head_dim")]


class as2d_tree_rows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_type", ctypes.c_int32), ("n_q", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("kv_len", ctypes.c_void_p),
                ("max_len", ctypes.c_int32), ("rows", ctypes.c_void_p),
                ("visible", ctypes.c_void_p), ("scale", ctypes.c_float)]


class as2d_cache4(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k", "k_scale", "v", "v_scale")] + \
               [(n, ctypes.c_int32) for n in ("n_layers", "batch", "n_kv", "capacity", "head_dim")]


class as2d_new_rows(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("type", ctypes.c_int32), ("n_q", ctypes.c_int32), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("kv_len", ctypes.c_void_p), ("rows", ctypes.c_void_p),
                ("positions", ctypes.c_void_p), ("q_norm", ctypes.c_void_p),
                ("k_norm", ctypes.c_void_p), ("eps", ctypes.c_float), ("theta", ctypes.c_float),
                ("rotary", ctypes.c_int32)]


class as2d_session_spec(ctypes.Structure):
    _fields_ = [("target", ctypes.c_void_p), ("drafter", ctypes.c_void_p),
                ("buf", ctypes.c_void_p), ("script", ctypes.c_void_p),
                ("n_script", ctypes.c_int32), ("b", ctypes.c_int32),
                ("publish_every", ctypes.c_int32), ("n_commit", ctypes.c_int32),
                ("overlapped", ctypes.c_int32), ("target_stream", ctypes.c_void_p),
                ("drafter_stream", ctypes.c_void_p), ("cpu_drafter", ctypes.c_void_p)]


class as2d_session_stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("T", "D", "V", "O", "H")] + \
               [(n, ctypes.c_int32) for n in ("rounds", "alone_rounds", "committed", "accepted",
                                              "producer_steps", "published")]


_P = ctypes.c_void_p
_S = ctypes.c_int32
_lib.as2d_model_load.argtypes = [ctypes.POINTER(as2d_config), ctypes.POINTER(as2d_weights),
                                 ctypes.POINTER(ctypes.c_void_p)]
_lib.as2d_model_load.restype = _S
_lib.as2d_kv_init_prefilled.argtypes = [_P, ctypes.c_int32, _P, ctypes.c_int32, _P, _P, _P,
                                        ctypes.POINTER(ctypes.c_void_p)]
_lib.as2d_kv_init_prefilled.restype = _S
_lib.as2d_verify_block.argtypes = [_P, _P, _P, ctypes.POINTER(as2d_verify_out), _P]
_lib.as2d_verify_block.restype = _S
_lib.as2d_decode_step.argtypes = [_P, ctypes.POINTER(as2d_verify_out), _P]
_lib.as2d_decode_step.restype = _S
_lib.as2d_kv_rollback.argtypes = [_P, _P, _P, _P]
_lib.as2d_kv_rollback.restype = _S
_lib.as2d_kv_read_state.argtypes = [_P, _P, _P, _P]
_lib.as2d_kv_read_state.restype = _S
_lib.as2d_kv_device_state.argtypes = [_P, ctypes.POINTER(ctypes.c_void_p),
                                      ctypes.POINTER(ctypes.c_void_p)]
_lib.as2d_kv_device_state.restype = _S
_lib.as2d_kv_check.argtypes = [_P, _P]
_lib.as2d_kv_check.restype = _S
_lib.as2d_kv_free.argtypes = [_P]
_lib.as2d_kv_free.restype = None
_lib.as2d_model_free.argtypes = [_P]
_lib.as2d_model_free.restype = None
_lib.as2d_kv_profile.argtypes = [_P, ctypes.c_int32]
_lib.as2d_kv_profile.restype = _S
_lib.as2d_kv_profile_read.argtypes = [_P, ctypes.POINTER(ctypes.c_int32),
                                      ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(ctypes.c_int64)]
_lib.as2d_kv_profile_read.restype = _S
_lib.as2d_decode_step_static.argtypes = [_P, _P, _P, ctypes.c_int32, _P, _P, _P, _P, _P, _P]
_lib.as2d_kv_set_wait_limit.argtypes = [_P, ctypes.c_uint64]
_lib.as2d_kv_set_wait_limit.restype = _S
_lib.as2d_decode_step_static.restype = _S
_lib.as2d_cbuf_create.argtypes = [_S, ctypes.POINTER(ctypes.c_void_p)]
_lib.as2d_cbuf_publish.argtypes = [_P, _P, _S, ctypes.POINTER(as2d_source_record)]
_lib.as2d_cbuf_candidates.argtypes = [_P, _S, _P, ctypes.POINTER(ctypes.c_int32)]
_lib.as2d_cbuf_after_call.argtypes = [_P, _S, _S, _S]
_lib.as2d_cbuf_state.argtypes = [_P, _P, _P, _P]
_lib.as2d_cbuf_source_of.argtypes = [_P, _S, ctypes.POINTER(as2d_source_record)]
_lib.as2d_cbuf_held.argtypes = [_P, _P, _P]
_lib.as2d_cbuf_held.restype = _S
_lib.as2d_cbuf_free.argtypes = [_P]
_lib.as2d_cbuf_free.restype = None
_lib.as2d_verify_from_buffers.argtypes = [_P, _P, _S, _P, _P, _P, _P]
for _n in ("as2d_cbuf_create", "as2d_cbuf_publish", "as2d_cbuf_candidates",
           "as2d_cbuf_after_call", "as2d_cbuf_state", "as2d_cbuf_source_of",
           "as2d_verify_from_buffers"):
    getattr(_lib, _n).restype = _S
_lib.as2d_interval_accounting.argtypes = [_P, _S, _P, _S, ctypes.c_double, _P]
_lib.as2d_interval_accounting.restype = _S
_lib.as2d_session_run.argtypes = [ctypes.POINTER(as2d_session_spec), _P,
                                  ctypes.POINTER(as2d_session_stats)]
_lib.as2d_session_run.restype = _S
_lib.as2d_budget_select.argtypes = [_P, _P, _P, _P, _P, _S, _S, _S, _S, _P, _P, _P]
_lib.as2d_budget_select.restype = _S
_lib.as2d_model_set_sm_budget.argtypes = [_P, _S]
_lib.as2d_model_set_sm_budget.restype = _S
_lib.as2d_prefill.argtypes = [_P, _P, _S, _P, _P]
_lib.as2d_prefill.restype = _S
_lib.as2d_cpu_decoder_create.argtypes = [ctypes.POINTER(as2d_config), ctypes.POINTER(as2d_weights),
                                         _S, _S, _S, ctypes.POINTER(ctypes.c_void_p)]
_lib.as2d_cpu_decoder_step.argtypes = [_P, ctypes.POINTER(ctypes.c_int32)]
_lib.as2d_cpu_decoder_logits.argtypes = [_P, _P]
_lib.as2d_cpu_decoder_reset.argtypes = [_P, _S, _S]
_lib.as2d_cpu_decoder_free.argtypes = [_P]
_lib.as2d_cpu_decoder_free.restype = None
for _n in ("as2d_cpu_decoder_create", "as2d_cpu_decoder_step", "as2d_cpu_decoder_logits",
           "as2d_cpu_decoder_reset"):
    getattr(_lib, _n).restype = _S
# (rows are described by their structure, or by its bytes)
_CACHE, _ROWS, _I64 = ctypes.POINTER(as2d_cache), _P, ctypes.c_int64
_lib.as2d_tree_attention_workspace.argtypes = [_CACHE, ctypes.POINTER(_I64)]
_lib.as2d_tree_attention.argtypes = [_CACHE, _S, _ROWS, _P, _P, _P, _I64, _P, _P]
_lib.as2d_attention_weights.argtypes = [_CACHE, _S, _ROWS, _P, _P, _P, _P]
_lib.as2d_cache_evict_workspace.argtypes = [_CACHE, ctypes.POINTER(_I64)]
_lib.as2d_cache_evict.argtypes = [_CACHE, _P, _P, _P, _S, _P, _I64, _P]
_CACHE4, _NEW = ctypes.POINTER(as2d_cache4), _P
_lib.as2d_cache_append.argtypes = [_CACHE, _S, _NEW, _P, _P, _P]
_lib.as2d_cache4_append.argtypes = [_CACHE4, _S, _NEW, _P, _P, _P]
_lib.as2d_cache4_write.argtypes = [_CACHE4, _CACHE, _S, _P, _P, _S, _P, _P]
_lib.as2d_cache4_read.argtypes = [_CACHE4, _CACHE, _S, _P, _P, _S, _P, _P]
_lib.as2d_cache4_attention_workspace.argtypes = [_CACHE4, ctypes.POINTER(_I64)]
_lib.as2d_cache4_attention.argtypes = [_CACHE4, _S, _ROWS, _P, _P, _P, _I64, _P, _P]
_lib.as2d_prompt_attention_workspace.argtypes = [_CACHE, ctypes.POINTER(_I64)]
_lib.as2d_prompt_attention.argtypes = [_CACHE, _S, _ROWS, _P, _P, _P, _I64, _P, _P]
_lib.as2d_token_probs.argtypes = [_P, _S, _S, ctypes.c_float, _P, _P]
_lib.as2d_accept_sampled.argtypes = [_P, _P, _P, _P, _S, _S, _P, _P, _P, _P]
_lib.as2d_verify_tree.argtypes = [_P, _P, _P, _P, ctypes.POINTER(as2d_verify_out), _P, _P]
_lib.as2d_verify_sampled.argtypes = [_P, _P, _P, _P, _P, ctypes.c_float,
                                     ctypes.POINTER(as2d_verify_out), _P, _P]
_lib.as2d_kv_track_weights.argtypes = [_P, _P]
_lib.as2d_kv_evict.argtypes = [_P, _P, _S, _P]
for _n in ("as2d_verify_tree", "as2d_verify_sampled", "as2d_kv_track_weights", "as2d_kv_evict",
           "as2d_tree_attention_workspace", "as2d_tree_attention", "as2d_attention_weights",
           "as2d_cache_evict_workspace", "as2d_cache_evict", "as2d_token_probs",
           "as2d_accept_sampled", "as2d_cache_append", "as2d_cache4_append", "as2d_cache4_write",
           "as2d_cache4_read", "as2d_cache4_attention_workspace", "as2d_cache4_attention",
           "as2d_prompt_attention_workspace", "as2d_prompt_attention"):
    getattr(_lib, _n).restype = _S
_lib.as2d_last_error.argtypes = []
_lib.as2d_last_error.restype = ctypes.c_char_p


class AS2DError(RuntimeError):
    def __init__(self, status, where):
        msg = _lib.as2d_last_error().decode(errors="replace")
        super().__init__(f"{where} returned {status}: {msg}")
        self.status = status


def _check(status, where):
    if status != AS2D_OK:
        raise AS2DError(status, where)
    return status


def _i32_array(values):
    arr = (ctypes.c_int32 * len(values))(*[int(v) for v in values])
    return arr


# ---- the C entry points, one wrapper each -------------------------------------

def as2d_last_error():
    return _lib.as2d_last_error().decode(errors="replace")


def as2d_model_load(cfg, weights_ptrs, n_layers):
    """cfg: as2d_config; weights_ptrs: dict name -> device pointer (int) for
    embed/final_norm/lm_head and name -> list of n_layers pointers for the
    per-layer tensors.  Returns (status, model handle)."""
    keep = []
    w = as2d_weights()
    for name in ("embed", "final_norm", "lm_head"):
        setattr(w, name, int(weights_ptrs[name]))
    for name in ("attn_norm", "w_q", "w_k", "w_v", "w_o", "mlp_norm", "w_gate",
                 "w_up", "w_down"):
        arr = (ctypes.c_void_p * n_layers)(*[int(p) for p in weights_ptrs[name]])
        keep.append(arr)
        setattr(w, name, ctypes.cast(arr, ctypes.c_void_p).value)
    out = ctypes.c_void_p()
    st = _lib.as2d_model_load(ctypes.byref(cfg), ctypes.byref(w), ctypes.byref(out))
    return st, out.value


def as2d_kv_init_prefilled(model, batch, kv_len, capacity, k_cache_ptr, v_cache_ptr,
                           root_tokens):
    out = ctypes.c_void_p()
    st = _lib.as2d_kv_init_prefilled(_P(model), int(batch), _i32_array(kv_len),
                                     int(capacity), _P(int(k_cache_ptr)),
                                     _P(int(v_cache_ptr)), _i32_array(root_tokens),
                                     ctypes.byref(out))
    return st, out.value


def make_verify_out(n_accepted_ptr, correction_ptr, greedy_ptr=0, logits_ptr=0):
    return as2d_verify_out(int(n_accepted_ptr) or None, int(correction_ptr) or None,
                           int(greedy_ptr) or None, int(logits_ptr) or None)


def as2d_verify_block(kv, candidates_ptr, k, out, stream=0):
    return _lib.as2d_verify_block(_P(kv), _P(int(candidates_ptr) or None), _i32_array(k),
                                  ctypes.byref(out), _P(int(stream) or None))


def as2d_decode_step(kv, out, stream=0):
    return _lib.as2d_decode_step(_P(kv), ctypes.byref(out), _P(int(stream) or None))


def as2d_kv_rollback(kv, new_len, new_root, stream=0):
    return _lib.as2d_kv_rollback(_P(kv), _i32_array(new_len), _i32_array(new_root),
                                 _P(int(stream) or None))


def as2d_kv_read_state(kv, batch, stream=0):
    ln = (ctypes.c_int32 * batch)()
    rt = (ctypes.c_int32 * batch)()
    st = _lib.as2d_kv_read_state(_P(kv), ln, rt, _P(int(stream) or None))
    return st, list(ln), list(rt)


def as2d_kv_device_state(kv):
    ln = ctypes.c_void_p()
    rt = ctypes.c_void_p()
    st = _lib.as2d_kv_device_state(_P(kv), ctypes.byref(ln), ctypes.byref(rt))
    return st, ln.value, rt.value


def as2d_kv_check(kv, stream=0):
    return _lib.as2d_kv_check(_P(kv), _P(int(stream) or None))


def as2d_kv_free(kv):
    _lib.as2d_kv_free(_P(kv))


def as2d_model_free(model):
    _lib.as2d_model_free(_P(model))


def as2d_kv_profile(kv, kernel_class):
    return _lib.as2d_kv_profile(_P(kv), int(kernel_class))


def as2d_kv_profile_read(kv):
    n = ctypes.c_int32()
    ms = ctypes.c_double()
    alln = ctypes.c_int64()
    st = _lib.as2d_kv_profile_read(_P(kv), ctypes.byref(n), ctypes.byref(ms), ctypes.byref(alln))
    return st, n.value, ms.value, alln.value


def as2d_decode_step_static(model, k_cache_ptr, v_cache_ptr, capacity, len_ptr, root_ptr,
                            correction_ptr, logits_ptr=0, error_bits_ptr=0, stream=0):
    """Single-request decode step whose working memory is the library's fixed
    array (no allocation); see include/as2d.h."""
    return _lib.as2d_decode_step_static(_P(model), _P(int(k_cache_ptr)), _P(int(v_cache_ptr)),
                                        int(capacity), _P(int(len_ptr)), _P(int(root_ptr)),
                                        _P(int(correction_ptr)), _P(int(logits_ptr) or None),
                                        _P(int(error_bits_ptr) or None),
                                        _P(int(stream) or None))


def as2d_cbuf_create(window):
    h = ctypes.c_void_p()
    st = _lib.as2d_cbuf_create(window, ctypes.byref(h))
    return st, h.value


def as2d_cbuf_publish(buf, tokens, record):
    arr = _i32_array(tokens) if len(tokens) else None
    return _lib.as2d_cbuf_publish(buf, arr, len(tokens),
                                  ctypes.byref(record) if record is not None else None)


def as2d_cbuf_candidates(buf, b):
    arr = (ctypes.c_int32 * max(b, 1))()
    k = ctypes.c_int32(-1)
    st = _lib.as2d_cbuf_candidates(buf, b, arr, ctypes.byref(k))
    return st, list(arr[:max(k.value, 0)])


def as2d_cbuf_after_call(buf, k, n_accepted, correction):
    return _lib.as2d_cbuf_after_call(buf, k, n_accepted, correction)


def as2d_cbuf_state(buf):
    r, c, m = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    st = _lib.as2d_cbuf_state(buf, ctypes.byref(r), ctypes.byref(c), ctypes.byref(m))
    return st, r.value, c.value, m.value


def as2d_cbuf_source_of(buf, position):
    rec = as2d_source_record()
    st = _lib.as2d_cbuf_source_of(buf, position, ctypes.byref(rec))
    return st, rec


def as2d_cbuf_free(buf):
    _lib.as2d_cbuf_free(buf)


def as2d_verify_from_buffers(kv, bufs, b, batch, stream=0):
    """Returns (status, k_used, committed lists)."""
    hb = (ctypes.c_void_p * batch)(*bufs)
    k_used = (ctypes.c_int32 * batch)()
    comm = (ctypes.c_int32 * (batch * (b + 1)))()
    ncomm = (ctypes.c_int32 * batch)()
    st = _lib.as2d_verify_from_buffers(kv, hb, b, k_used, comm, ncomm, stream)
    rows = [list(comm[r * (b + 1): r * (b + 1) + ncomm[r]]) for r in range(batch)]
    return st, list(k_used), rows


def as2d_interval_accounting(p, v, T):
    """p, v: lists of (start, end).  Returns (status, [D, V, O, H, T])."""
    pa = (ctypes.c_double * max(2 * len(p), 1))(*[x for iv in p for x in iv])
    va = (ctypes.c_double * max(2 * len(v), 1))(*[x for iv in v for x in iv])
    out = (ctypes.c_double * 5)()
    st = _lib.as2d_interval_accounting(pa, len(p), va, len(v), T, out)
    return st, list(out)


def as2d_session_run(spec, n_commit, b):
    """Returns (status, committed list, stats dict)."""
    comm = (ctypes.c_int32 * (n_commit + AS2D_MAX_K + 1))()
    stats = as2d_session_stats()
    st = _lib.as2d_session_run(ctypes.byref(spec), comm, ctypes.byref(stats))
    d = {n: getattr(stats, n) for n, _ in as2d_session_stats._fields_}
    return st, list(comm[:max(stats.committed, 0)]), d


class CpuDecoder:
    """Owns an as2d_cpu_decoder built from host fp32 weights: `host` maps the
    names of as2d_weights to float32 numpy arrays (per-layer names to lists)."""

    def __init__(self, shape, host, capacity, threads, root):
        import numpy as np
        self._keep = {k: ([np.ascontiguousarray(a, dtype=np.float32) for a in v]
                          if isinstance(v, list) else np.ascontiguousarray(v, dtype=np.float32))
                      for k, v in host.items()}
        w = as2d_weights()
        for name in ("embed", "final_norm", "lm_head"):
            setattr(w, name, self._keep[name].ctypes.data)
        self._arrs = []
        for name in ("attn_norm", "w_q", "w_k", "w_v", "w_o", "mlp_norm", "w_gate", "w_up",
                     "w_down"):
            arr = (ctypes.c_void_p * shape.n_layers)(*[a.ctypes.data for a in self._keep[name]])
            self._arrs.append(arr)
            setattr(w, name, ctypes.cast(arr, ctypes.c_void_p))
        cfg = as2d_config(shape.n_layers, shape.hidden, shape.n_q, shape.n_kv, shape.head_dim,
                          shape.ffn, shape.vocab, float(shape.rope_theta), float(shape.rms_eps))
        h = ctypes.c_void_p()
        _check(_lib.as2d_cpu_decoder_create(ctypes.byref(cfg), ctypes.byref(w), capacity, threads,
                                            root, ctypes.byref(h)), "as2d_cpu_decoder_create")
        self.handle = h.value
        self.vocab = shape.vocab
        self._keep = None  # copied by the library

    def step(self):
        t = ctypes.c_int32()
        _check(_lib.as2d_cpu_decoder_step(self.handle, ctypes.byref(t)), "as2d_cpu_decoder_step")
        return t.value

    def logits(self):
        import numpy as np
        out = np.empty(self.vocab, dtype=np.float32)
        _check(_lib.as2d_cpu_decoder_logits(self.handle, out.ctypes.data),
               "as2d_cpu_decoder_logits")
        return out

    def reset(self, length, root):
        _check(_lib.as2d_cpu_decoder_reset(self.handle, length, root), "as2d_cpu_decoder_reset")

    def close(self):
        if self.handle:
            _lib.as2d_cpu_decoder_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def session_run(target, drafter, buf, script, b, n_commit, overlapped, publish_every=8,
                target_stream=0, drafter_stream=0, cpu_drafter=None):
    """Run a producer/verifier session (as2d_session_run) on State objects and
    a CandidateBuffer; returns (committed tokens, stats dict)."""
    arr = _i32_array(script) if len(script) else None
    spec = as2d_session_spec(target.handle, drafter.handle if drafter is not None else None,
                             buf.handle, ctypes.cast(arr, ctypes.c_void_p) if arr else None,
                             len(script), b, publish_every, n_commit, int(bool(overlapped)),
                             target_stream, drafter_stream,
                             cpu_drafter.handle if cpu_drafter is not None else None)
    st, comm, stats = as2d_session_run(spec, n_commit, b)
    _check(st, "as2d_session_run")
    return comm, stats


def as2d_budget_select(cost_us, traces, n_commit, window, b_max):
    """cost_us: AS2D_MAX_K + 1 mean call times by k; traces: list of
    (reference text, producer text).  Returns (status, best b, tok/s per b,
    calls per b)."""
    cost = (ctypes.c_double * (AS2D_MAX_K + 1))(*[float(c) for c in cost_us])
    refs = [int(t) for r, _ in traces for t in r]
    prods = [int(t) for _, p in traces for t in p]
    ra = _i32_array(refs or [0])
    pa = _i32_array(prods or [0])
    rl = _i32_array([len(r) for r, _ in traces] or [0])
    pl = _i32_array([len(p) for _, p in traces] or [0])
    tok_s = (ctypes.c_double * (max(b_max, 0) + 1))()
    calls = (ctypes.c_int32 * (max(b_max, 0) + 1))()
    best = ctypes.c_int32(-1)
    st = _lib.as2d_budget_select(cost, ra, rl, pa, pl, len(traces), n_commit, window, b_max,
                                 tok_s, calls, ctypes.byref(best))
    return st, best.value, list(tok_s), list(calls)


def exported_symbols():
    """Names of include/as2d.h's entry points that the loaded library exports."""
    return [n for n in EXPORTED if hasattr(_lib, n)]


# ---- thin owners of the handles (marshalling only) ---------------------------

class Model:
    """Owns an as2d_model.  `shape` has the fields of as2d_config
    (n_layers, hidden, n_q, n_kv, head_dim, ffn, vocab, rope_theta, rms_eps);
    `pointers` maps weight names to device pointers (see as2d_model_load)."""

    def __init__(self, shape, pointers):
        self.shape = shape
        self.cfg = as2d_config(shape.n_layers, shape.hidden, shape.n_q, shape.n_kv,
                               shape.head_dim, shape.ffn, shape.vocab,
                               float(shape.rope_theta), float(shape.rms_eps))
        st, h = as2d_model_load(self.cfg, pointers, shape.n_layers)
        _check(st, "as2d_model_load")
        self.handle = h

    def set_sm_budget(self, n_sms):
        _check(_lib.as2d_model_set_sm_budget(self.handle, int(n_sms)), "as2d_model_set_sm_budget")

    def close(self):
        if self.handle:
            as2d_model_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class CandidateBuffer:
    """Owns an as2d_cbuf: one request's published candidates, read cursor and
    alignment state (host side)."""

    def __init__(self, window=8):
        st, h = as2d_cbuf_create(window)
        _check(st, "as2d_cbuf_create")
        self.handle = h

    def publish(self, tokens, request=0, source=0, producer=0, offset=0, time=0.0,
                confidence=None):
        rec = as2d_source_record(request, source, producer, offset, time,
                                 0.0 if confidence is None else confidence,
                                 0 if confidence is None else 1)
        _check(as2d_cbuf_publish(self.handle, list(tokens), rec), "as2d_cbuf_publish")

    def candidates(self, b):
        st, toks = as2d_cbuf_candidates(self.handle, b)
        _check(st, "as2d_cbuf_candidates")
        return toks

    def after_call(self, k, n_accepted, correction):
        _check(as2d_cbuf_after_call(self.handle, k, n_accepted, correction),
               "as2d_cbuf_after_call")

    def state(self):
        st, ready, cursor, mode = as2d_cbuf_state(self.handle)
        _check(st, "as2d_cbuf_state")
        return ready, cursor, CBUF_MODES[mode]

    def held(self):
        """(tokens, batch records) the buffer still holds."""
        t, r = ctypes.c_int32(), ctypes.c_int32()
        _check(_lib.as2d_cbuf_held(self.handle, ctypes.byref(t), ctypes.byref(r)), "as2d_cbuf_held")
        return t.value, r.value

    def source_of(self, position):
        st, rec = as2d_cbuf_source_of(self.handle, position)
        _check(st, "as2d_cbuf_source_of")
        return {"request": rec.request, "source": rec.source, "producer": rec.producer,
                "offset": rec.offset, "time": rec.time,
                "confidence": rec.confidence if rec.has_confidence else None}

    def close(self):
        if self.handle:
            as2d_cbuf_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class State:
    """Owns an as2d_kv bound to caller caches (torch tensors kept alive here)."""

    def __init__(self, model, kv_len, capacity, k_cache, v_cache, roots):
        self.model = model
        self.batch = len(kv_len)
        self._caches = (k_cache, v_cache)
        self._places = model.cfg.n_layers * self.batch * model.cfg.n_kv_heads * capacity
        st, h = as2d_kv_init_prefilled(model.handle, self.batch, kv_len, capacity,
                                       k_cache.data_ptr(), v_cache.data_ptr(), roots)
        _check(st, "as2d_kv_init_prefilled")
        self.handle = h

    def verify(self, candidates, k, n_accepted, correction, greedy=None, logits=None,
               stream=0):
        out = make_verify_out(n_accepted.data_ptr(), correction.data_ptr(),
                              greedy.data_ptr() if greedy is not None else 0,
                              logits.data_ptr() if logits is not None else 0)
        cptr = candidates.data_ptr() if candidates is not None and candidates.numel() else 0
        _check(as2d_verify_block(self.handle, cptr, k, out, stream), "as2d_verify_block")

    def decode(self, n_accepted, correction, greedy=None, logits=None, stream=0):
        out = make_verify_out(n_accepted.data_ptr(), correction.data_ptr(),
                              greedy.data_ptr() if greedy is not None else 0,
                              logits.data_ptr() if logits is not None else 0)
        _check(as2d_decode_step(self.handle, out, stream), "as2d_decode_step")

    def _counts(self, values, name):
        if len(values) != self.batch:
            raise ValueError(f"{name} must name {self.batch} requests")
        return _int32s(values, name)

    def _address(self, t, name, dtype, least):
        """Device address of a contiguous tensor of `least` elements or more on the caches' device
        (None: NULL)."""
        if t is None:
            return None
        if str(t.dtype) != dtype:
            raise TypeError(f"{name} must be a tensor of {dtype}")
        if t.get_device() != self._caches[0].get_device():
            raise ValueError(f"{name} must be on the caches' device")
        if not t.is_contiguous() or t.numel() < least:
            raise ValueError(f"{name} must be contiguous, of {least} elements")
        return t.data_ptr()

    def verify_tree(self, candidates, parents, k, n_accepted, correction, greedy=None, logits=None,
                    path=None, stream=0):
        """as2d_verify_tree: device int32 candidates and parents, packed."""
        counts, total = self._counts(k, "k"), sum(k)
        rows, i32, at = total + self.batch, "torch.int32", self._address
        out = make_verify_out(at(n_accepted, "n_accepted", i32, self.batch),
                              at(correction, "correction", i32, self.batch), at(greedy, "greedy", i32, rows) or 0,
                              at(logits, "logits", "torch.float32", rows * self.model.cfg.vocab) or 0)
        some = candidates is not None and candidates.numel()
        _check(_lib.as2d_verify_tree(
            self.handle, at(candidates if some else None, "candidates", i32, total),
            at(parents if some else None, "parents", i32, total), counts, ctypes.byref(out),
            at(path, "path", i32, self.batch * AS2D_MAX_K), stream), "as2d_verify_tree")

    def verify_sampled(self, candidates, k, u, temperature, probs, n_accepted, correction,
                       draft_probs=None, greedy=None, stream=0):
        """as2d_verify_sampled: u [rows] and probs [rows, vocab] device float."""
        counts, total, vocab = self._counts(k, "k"), sum(k), self.model.cfg.vocab
        rows, i32, f32, at = total + self.batch, "torch.int32", "torch.float32", self._address
        out = make_verify_out(at(n_accepted, "n_accepted", i32, self.batch),
                              at(correction, "correction", i32, self.batch), at(greedy, "greedy", i32, rows) or 0)
        some = candidates is not None and candidates.numel()
        _check(_lib.as2d_verify_sampled(
            self.handle, at(candidates if some else None, "candidates", i32, total), counts,
            at(draft_probs if some else None, "draft_probs", f32, total * vocab), at(u, "u", f32, rows),
            temperature, ctypes.byref(out), at(probs, "probs", f32, rows * vocab), stream), "as2d_verify_sampled")

    def track_weights(self, weights):
        """as2d_kv_track_weights: a device float tensor (kept alive here) or None."""
        _check(_lib.as2d_kv_track_weights(
            self.handle, self._address(weights, "weights", "torch.float32", self._places)), "as2d_kv_track_weights")
        self._weights = weights

    def evict(self, keep, recent=0, stream=0):
        _check(_lib.as2d_kv_evict(self.handle, self._counts(keep, "keep"), _int32s((recent,), "recent")[0], stream),
               "as2d_kv_evict")

    def verify_from_buffers(self, bufs, b, stream=0):
        """One verification call with candidates from CandidateBuffer objects
        (one per request); returns (k_used, committed token lists)."""
        st, k_used, rows = as2d_verify_from_buffers(
            self.handle, [x.handle for x in bufs], b, self.batch, stream)
        _check(st, "as2d_verify_from_buffers")
        return k_used, rows

    def prefill(self, tokens, first_token=None, stream=0):
        """as2d_prefill: tokens and first_token are device int32 tensors."""
        _check(_lib.as2d_prefill(self.handle, tokens.data_ptr(), tokens.numel(),
                                 first_token.data_ptr() if first_token is not None else None,
                                 stream), "as2d_prefill")

    def rollback(self, new_len, new_root, stream=0):
        _check(as2d_kv_rollback(self.handle, new_len, new_root, stream), "as2d_kv_rollback")

    def read_state(self, stream=0):
        st, ln, rt = as2d_kv_read_state(self.handle, self.batch, stream)
        _check(st, "as2d_kv_read_state")
        return ln, rt

    def device_state(self):
        st, ln, rt = as2d_kv_device_state(self.handle)
        _check(st, "as2d_kv_device_state")
        return ln, rt

    def profile(self, kernel_class):
        cls = KERNEL_CLASSES[kernel_class] if isinstance(kernel_class, str) else kernel_class
        _check(as2d_kv_profile(self.handle, -1 if cls is None else cls), "as2d_kv_profile")

    def profile_read(self):
        st, n, ms, alln = as2d_kv_profile_read(self.handle)
        _check(st, "as2d_kv_profile_read")
        return n, ms, alln

    def set_wait_limit(self, ns):
        _check(_lib.as2d_kv_set_wait_limit(self.handle, int(ns)), "as2d_kv_set_wait_limit")

    def check(self, stream=0):
        _check(as2d_kv_check(self.handle, stream), "as2d_kv_check")

    def close(self):
        if self.handle:
            as2d_kv_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- operators on tensors ------------------------------------------------------
#
# A call is enqueued on `stream` (a cudaStream_t, 0 for the legacy default stream), on torch's
# current stream unless one is given.  A result that the call makes itself belongs to that
# stream, as a tensor that torch makes there would.

def _int32s(values, name):
    """A C array of Python integers; ctypes itself takes those beyond 32 bits modulo 2^32."""
    values = list(values)
    array = (ctypes.c_int32 * len(values))(*values)
    if array[:] != values:
        raise ValueError(f"{name} must be of 32 bits")
    return array


def _stream_reader(torch):
    """A function that gives torch's current stream of a device as a cudaStream_t."""
    return (getattr(torch._C, "_cuda_getCurrentRawStream", None) or
            (lambda device: torch.cuda.current_stream(device).cuda_stream))


def _new_on(stream, device, like, shape):
    """An uninitialised tensor of like's type that belongs to `stream`."""
    import torch
    of = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.stream(of):
        return like.new_empty(shape)


def _tensor(t, name, device, dtypes, shape=None, contiguous=True):
    """Checks a CUDA tensor argument and returns its device address."""
    if getattr(t, "dtype", None) not in dtypes:
        raise TypeError(f"{name} must be a tensor of {' or '.join(map(str, dtypes))}")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on the current CUDA device")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _address(t, name, device, dtype, shape):
    """The same of a contiguous tensor of one type and shape: the common case in one
    expression, as a small call's time is the host's."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    return _tensor(t, name, device, (dtype,), shape)


def _packer(structure, layout):
    """A function that gives the bytes of a structure's fields, in a third of the time that the
    structure itself takes; what it refuses is left to that (numbers beyond 32 bits, errors)."""
    packer = struct.Struct(layout)
    assert packer.size == ctypes.sizeof(structure)
    pack = packer.pack

    def fields(*values):
        try:
            return pack(*values)
        except (struct.error, OverflowError):
            return bytes(structure(*values))
    return fields


_TREE_ROWS = _packer(as2d_tree_rows, "@PiiqPiPPf4x")
_NEW_ROWS = _packer(as2d_new_rows, "@PPPiiqqqPPPPPffi4x")


class _CacheCalls:
    """What the caches below share: checks of a call's arguments, the workspace and its stream."""

    def _set_up(self, c, shape, device, k):
        import torch
        self._c, self.shape, self._on = c, shape, device
        self._current = torch.cuda.current_device
        self._ref = ctypes.byref(self._c)
        self._per_request, self._counts_type = shape[1:2], ctypes.c_int32 * shape[1]
        self._bf16, self._f32, self._i32, self._i64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
        self._mask = (torch.int64, torch.uint64)
        most, need = 0, _I64()
        for name in self._WORKSPACES:
            _check(getattr(_lib, name)(self._ref, ctypes.byref(need)), name)
            most = max(most, need.value)
        self._workspace = torch.empty(most, dtype=torch.uint8, device=k.device)
        self._current_stream = _stream_reader(torch)
        self._made_on = self._current_stream(device)

    def _enter(self, stream):
        """(device, torch's current stream, the call's stream) of a call."""
        device = self._current()
        if device != self._on:
            raise ValueError("the cache must be on the current CUDA device")
        current = self._current_stream(device)
        if stream is None and current != self._made_on:
            import torch  # torch's allocator is told of a use on another stream than the workspace's own
            self._workspace.record_stream(torch.cuda.current_stream(device))
        return device, current, current if stream is None else stream

    def _counts(self, values, name):
        if len(values) != self.shape[1]:
            raise ValueError(f"{name} must name {self.shape[1]} requests")
        array = self._counts_type(*values)
        if array[:] != (values if type(values) is list else list(values)):
            raise ValueError(f"{name} must be of 32 bits")
        return array

    def _rows(self, device, q, kv_len, rows, visible, scale, layer, max_len):
        d = self.shape[4]
        if abs(layer) >> 31 or abs(max_len) >> 31:
            raise ValueError("layer and max_len must be of 32 bits")
        at = _tensor(q, "q", device, (self._bf16, self._f32), None, False)
        shape = q.shape
        n_q = shape[1] if len(shape) == 3 else 0
        if n_q == 0 or shape[2] != d or q.stride()[1:] != (d, 1):
            raise ValueError(f"q must be [rows, n_q, {d}] with contiguous rows")
        n = shape[0]
        host_rows = self._counts(rows, "rows")
        if n != sum(rows):
            raise ValueError("q must have as many rows as the requests together")
        if visible is not None:
            if visible.dtype is self._i64:
                visible = _address(visible, "visible", device, self._i64, shape[:1])
            else:
                visible = _tensor(visible, "visible", device, self._mask, shape[:1])
        r = _TREE_ROWS(
            at, AS2D_TYPE_BF16 if q.dtype is self._bf16 else AS2D_TYPE_F32, n_q,
            q.stride(0) if n > 1 else n_q * d,  # (the stride of a single row is not looked at)
            _address(kv_len, "kv_len", device, self._i32, self._per_request), max_len,
            ctypes.addressof(host_rows), visible or 0, d ** -0.5 if scale is None else scale)
        return r, host_rows  # (which the descriptor points to)

    def _attention(self, name, q, kv_len, rows, visible, scale, layer, max_len, out, lse, error_bits, stream,
                   space=None):
        device, current, stream = self._enter(stream)
        r, keep = self._rows(device, q, kv_len, rows, visible, scale, layer, max_len)
        shape = q.shape
        if out is None:
            out = q.new_empty(shape) if stream == current else _new_on(stream, device, q, shape)
        workspace = self._workspace if space is None else space(device, current, stream)
        st = getattr(_lib, name)(
            self._ref, layer, r, _address(out, "out", device, q.dtype, shape),
            None if lse is None else _address(lse, "lse", device, self._f32, shape[:2]),
            workspace.data_ptr(), workspace.numel(),
            None if error_bits is None else _tensor(error_bits, "error_bits", device, (self._i32,)),
            stream)
        if st:
            _check(st, name)
        return out

    def _check_new_rows(self, device, q, k, v):
        """What is wrong with the rows of an append."""
        n_kv, d = self.shape[2], self.shape[4]
        _tensor(q, "q", device, (self._bf16, self._f32), None, False)
        if q.dim() != 3 or q.shape[1] == 0 or q.shape[2] != d:
            raise ValueError(f"q must be [rows, n_q, {d}]")
        for t, name in ((k, "k"), (v, "v")):
            _tensor(t, name, device, (q.dtype,), (q.shape[0], n_kv, d), False)
        raise ValueError("the rows of q, k and v must be contiguous")

    def _append(self, name, q, k, v, kv_len, rows, layer, positions, q_norm, k_norm, eps, theta, rotary,
                out, error_bits, stream):
        device, current, stream = self._enter(stream)
        d = self.shape[4]
        # the common case in one expression, as a small call's time is the host's
        try:
            dtype, shape = q.dtype, q.shape
            n, n_q, _ = shape
            new = (n, self.shape[2], d)
            of_q, of_k, of_v = q.stride(), k.stride(), v.stride()
            good = (k.dtype is dtype and v.dtype is dtype and (dtype is self._bf16 or dtype is self._f32) and
                    n_q > 0 and shape[2] == d and k.shape == new and v.shape == new and
                    of_q[1] == of_k[1] == of_v[1] == d and of_q[2] == of_k[2] == of_v[2] == 1 and
                    q.get_device() == device and k.get_device() == device and v.get_device() == device)
        except (AttributeError, ValueError, IndexError):
            good = False
        if not good:
            self._check_new_rows(device, q, k, v)
        host_rows = self._counts(rows, "rows")
        if n != sum(rows):
            raise ValueError("q must have as many rows as the requests together")
        if n == 1:  # (the stride of a single row is not looked at)
            of_q, of_k, of_v = (n_q * d,), (new[1] * d,), (new[1] * d,)
        rotary = d if rotary is None else rotary
        if layer.bit_length() > 31 or rotary.bit_length() > 31:
            raise ValueError("layer and rotary must be of 32 bits")
        r = _NEW_ROWS(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), AS2D_TYPE_BF16 if dtype is self._bf16 else AS2D_TYPE_F32, n_q,
            of_q[0], of_k[0], of_v[0], _address(kv_len, "kv_len", device, self._i32, self._per_request),
            ctypes.addressof(host_rows),
            0 if positions is None else _address(positions, "positions", device, self._i32, (n,)),
            0 if q_norm is None else _address(q_norm, "q_norm", device, self._f32, (d,)),
            0 if k_norm is None else _address(k_norm, "k_norm", device, self._f32, (d,)), eps, theta, rotary)
        if out is None:
            out = q.new_empty(shape) if stream == current else _new_on(stream, device, q, shape)
        st = getattr(_lib, name)(
            self._ref, layer, r, _address(out, "out", device, dtype, shape),
            None if error_bits is None else _tensor(error_bits, "error_bits", device, (self._i32,)), stream)
        if st:
            _check(st, name)
        return out


class Cache(_CacheCalls):
    """A key/value cache of the caller's (two bf16 tensors [n_layers][batch][n_kv]
    [capacity][head_dim], kept alive here) with the workspace of the operators
    on it (prompts have one of their own, made with the first of them); see
    include/as2d.h, "Operators on caches and logits".  Calls on one
    Cache share the workspace, so calls that may overlap on the GPU (several
    streams, captured graphs) need a Cache each.  A Cache outlives the captured
    graphs that hold its calls, and calls enqueued on a stream that was given by
    its handle; those on torch's current stream may still run when it goes."""

    _WORKSPACES = ("as2d_tree_attention_workspace", "as2d_cache_evict_workspace")

    def __init__(self, k, v):
        import torch
        device = torch.cuda.current_device()
        kp = _tensor(k, "k", device, (torch.bfloat16,))
        if k.dim() != 5:
            raise ValueError("k must have shape [n_layers, batch, n_kv, capacity, head_dim]")
        vp = _tensor(v, "v", device, (torch.bfloat16,), k.shape)
        self.k, self.v = k, v
        self._set_up(as2d_cache(kp, vp, *k.shape), tuple(k.shape), device, k)
        self._prompts = None

    def _of_prompts(self, device, current, stream):
        """The prompts' workspace, twice the others': made with the first prompt, as its result would be."""
        if self._prompts is None:
            need = _I64()
            _check(_lib.as2d_prompt_attention_workspace(self._ref, ctypes.byref(need)), "as2d_prompt_attention_workspace")
            like, shape = self._workspace, (need.value,)
            self._prompts = like.new_empty(shape) if stream == current else _new_on(stream, device, like, shape)
            self._prompts_on = stream
        elif stream == current != self._prompts_on:
            import torch
            self._prompts.record_stream(torch.cuda.current_stream(device))
        return self._prompts

    def append(self, q, k, v, kv_len, rows, layer=0, positions=None, q_norm=None, k_norm=None, eps=1e-6,
               theta=1e6, rotary=None, out=None, error_bits=None, stream=None):
        """as2d_cache_append: q [rows, n_q, head_dim], k and v [rows, n_kv, head_dim]
        (parts of one tensor, if need be); rotary: the rotated dims (head_dim unless
        given).  Returns out, the queries (made like q unless given)."""
        return self._append("as2d_cache_append", q, k, v, kv_len, rows, layer, positions, q_norm, k_norm,
                            eps, theta, rotary, out, error_bits, stream)

    def prompt_attention(self, q, kv_len, rows, layer=0, scale=None, max_len=0, out=None, lse=None,
                         error_bits=None, stream=None):
        """as2d_prompt_attention; returns out (made like q unless given)."""
        return self._attention("as2d_prompt_attention", q, kv_len, rows, None, scale, layer, max_len, out, lse,
                               error_bits, stream, self._of_prompts)

    def tree_attention(self, q, kv_len, rows, visible=None, layer=0, scale=None, max_len=0, out=None,
                       lse=None, error_bits=None, stream=None):
        """as2d_tree_attention; returns out (made like q unless given)."""
        return self._attention("as2d_tree_attention", q, kv_len, rows, visible, scale, layer, max_len, out, lse,
                               error_bits, stream)

    def attention_weights(self, q, lse, weights, kv_len, rows, visible=None, layer=0, scale=None,
                          max_len=0, error_bits=None, stream=None):
        """as2d_attention_weights: adds to weights in place."""
        device, current, stream = self._enter(stream)
        r, keep = self._rows(device, q, kv_len, rows, visible, scale, layer, max_len)
        st = _lib.as2d_attention_weights(
            self._ref, layer, r, _address(lse, "lse", device, self._f32, q.shape[:2]),
            _address(weights, "weights", device, self._f32, self.shape[:4]),
            None if error_bits is None else _tensor(error_bits, "error_bits", device, (self._i32,)),
            stream)
        if st:
            _check(st, "as2d_attention_weights")

    def evict(self, weights, kv_len, keep, recent=0, stream=None):
        """as2d_cache_evict: cuts the cache, weights and kv_len in place."""
        device, _, stream = self._enter(stream)
        st = _lib.as2d_cache_evict(
            self._ref, _address(weights, "weights", device, self._f32, self.shape[:4]),
            _address(kv_len, "kv_len", device, self._i32, self._per_request),
            self._counts(keep, "keep"), _int32s((recent,), "recent")[0], self._workspace.data_ptr(),
            self._workspace.numel(), stream)
        if st:
            _check(st, "as2d_cache_evict")


class Cache4(_CacheCalls):
    """A key/value cache of the caller's in 4 bits (uint8 tensors k and v [n_layers][batch]
    [n_kv][capacity][head_dim / 2], k_scale and v_scale [..][head_dim / 16], kept alive
    here; as2d_cache4 in include/as2d.h has the format).  As Cache in what concerns
    streams and the workspace."""

    _WORKSPACES = ("as2d_cache4_attention_workspace",)

    def __init__(self, k, k_scale, v, v_scale):
        import torch
        device, u8 = torch.cuda.current_device(), (torch.uint8,)
        at = [_tensor(k, "k", device, u8)]
        if k.dim() != 5:
            raise ValueError("k must have shape [n_layers, batch, n_kv, capacity, head_dim / 2]")
        d = 2 * k.shape[4]
        scales = (*k.shape[:4], d // 16)
        for t, name, shape in ((k_scale, "k_scale", scales), (v, "v", k.shape), (v_scale, "v_scale", scales)):
            at.append(_tensor(t, name, device, u8, shape))
        self.k, self.k_scale, self.v, self.v_scale = k, k_scale, v, v_scale
        shape = (*k.shape[:4], d)
        self._set_up(as2d_cache4(*at, *shape), shape, device, k)

    def append(self, q, k, v, kv_len, rows, layer=0, positions=None, q_norm=None, k_norm=None, eps=1e-6,
               theta=1e6, rotary=None, out=None, error_bits=None, stream=None):
        """as2d_cache4_append; arguments as Cache.append."""
        return self._append("as2d_cache4_append", q, k, v, kv_len, rows, layer, positions, q_norm, k_norm,
                            eps, theta, rotary, out, error_bits, stream)

    def _convert(self, name, cache, end, start, layer, max_entries, error_bits, stream):
        device, _, stream = self._enter(stream)
        if not isinstance(cache, Cache):
            raise TypeError("cache must be a Cache")
        if cache._on != device:
            raise ValueError("both caches must be on the current CUDA device")
        layer = -1 if layer is None else layer
        if layer.bit_length() > 31 or max_entries.bit_length() > 31:
            raise ValueError("layer and max_entries must be of 32 bits")
        st = getattr(_lib, name)(
            self._ref, cache._ref, layer,
            None if start is None else _address(start, "start", device, self._i32, self._per_request),
            _address(end, "end", device, self._i32, self._per_request), max_entries,
            None if error_bits is None else _tensor(error_bits, "error_bits", device, (self._i32,)), stream)
        if st:
            _check(st, name)

    def write(self, cache, end, start=None, layer=None, max_entries=0, error_bits=None, stream=None):
        """as2d_cache4_write: entries [start, end) (int32 [batch], start 0 unless given) of
        a Cache into this one; every layer unless one is given."""
        self._convert("as2d_cache4_write", cache, end, start, layer, max_entries, error_bits, stream)

    def read(self, cache, end, start=None, layer=None, max_entries=0, error_bits=None, stream=None):
        """as2d_cache4_read: entries [start, end) of this cache into a Cache."""
        self._convert("as2d_cache4_read", cache, end, start, layer, max_entries, error_bits, stream)

    def tree_attention(self, q, kv_len, rows, visible=None, layer=0, scale=None, max_len=0, out=None,
                       lse=None, error_bits=None, stream=None):
        """as2d_cache4_attention; returns out (made like q unless given)."""
        return self._attention("as2d_cache4_attention", q, kv_len, rows, visible, scale, layer, max_len, out,
                               lse, error_bits, stream)


def token_probs(logits, temperature, out=None, stream=None):
    """as2d_token_probs of logits [rows, vocab]; returns out (made like logits
    unless given; may be logits)."""
    import torch
    device, shape = torch.cuda.current_device(), logits.shape
    at = _address(logits, "logits", device, torch.float32, shape)
    if len(shape) != 2:
        raise ValueError("logits must be [rows, vocab]")
    current = _stream_reader(torch)(device)
    if stream is None:
        stream = current
    if out is None:
        out = torch.empty_like(logits) if stream == current else _new_on(stream, device, logits, shape)
    st = _lib.as2d_token_probs(at, shape[0], shape[1], temperature,
                               _address(out, "out", device, torch.float32, shape), stream)
    if st:
        _check(st, "as2d_token_probs")
    return out


def accept_sampled(probs, candidates, k, u, n_accepted, token, draft_probs=None, stream=None):
    """as2d_accept_sampled: probs [sum (k + 1), vocab], candidates [sum k] (or
    None), k a list, u [sum (k + 1)], n_accepted and token [batch]."""
    import torch
    f32, i32 = torch.float32, torch.int32
    device, total, batch, shape = torch.cuda.current_device(), sum(k), len(k), probs.shape
    at = _address(probs, "probs", device, f32, shape)
    if len(shape) != 2 or shape[0] != total + batch:
        raise ValueError("probs must be [sum (k + 1), vocab]")
    if stream is None:
        stream = _stream_reader(torch)(device)
    st = _lib.as2d_accept_sampled(
        at, None if draft_probs is None or total == 0 else
        _address(draft_probs, "draft_probs", device, f32, (total, shape[1])),
        None if candidates is None or total == 0 else
        _address(candidates, "candidates", device, i32, (total,)), _int32s(k, "k"),
        batch, shape[1], _address(u, "u", device, f32, shape[:1]),
        _address(n_accepted, "n_accepted", device, i32, (batch,)),
        _address(token, "token", device, i32, (batch,)), stream)
    if st:
        _check(st, "as2d_accept_sampled")
