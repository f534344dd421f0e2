"""ctypes binding of libdd.so (include/dd.h).

Argument marshalling only: every step of the reverse step runs in the HIP
library.  Device buffers are torch tensors (data_ptr + the current HIP stream);
each wrapper checks that the tensors it hands over are contiguous, on the GPU and
large enough for the sizes it passes, so the library never reads or writes
outside an allocation.  The library must have been built in-tree
(python -m paper_2609_04010_amd.build); nothing falls back to another
implementation when it is missing.
"""
import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdd.so")

DD_BF16, DD_FP32 = 0, 1
DD_PRIOR_MASK, DD_PRIOR_UNIFORM = 0, 1
DD_NORM_LAYER, DD_NORM_RMS = 0, 1
DD_GUMBEL_GROUP = 256
DD_DEVERR_TOKEN = 1
DD_DEVERR_MASK = 2
DD_DEVERR_LOGITS = 4
DD_DEVERR_CACHE = 8
DD_DEVERR_SAMPLING = 16
DD_LOOP_POSTERIOR_PASS = 1
DD_LOOP_STORE_FREE = 2
ATTN_PATTERNS = {"bidirectional": 0, "causal": 1, "block_causal": 2, "draft_train": 3}
STATUS = {0: "DD_OK", 1: "DD_E_ARG", 2: "DD_E_SHAPE", 3: "DD_E_DTYPE", 4: "DD_E_WORKSPACE",
          5: "DD_E_HIP", 6: "DD_E_UNSUPPORTED", 7: "DD_E_DEVICE"}

EXPORTED = [
    "dd_param_count", "dd_param_tensor", "dd_param_bytes", "dd_workspace_bytes",
    "dd_loop_workspace_bytes", "dd_loop_workspace_layout", "dd_logits_ld", "dd_noise_width",
    "dd_status_str", "dd_last_error",
    "dd_workspace_reset", "dd_read_device_error", "dd_init_params", "dd_denoise_forward",
    "dd_attn_mask_build", "dd_denoise_forward_ex",
    "dd_posterior_sample", "dd_psi_posterior_sample", "dd_sample_loop", "dd_psi_sample_loop",
    "dd_gaussian_latent_argmax", "dd_spec_verify_workspace_bytes", "dd_spec_verify_noise_width",
    "dd_spec_verify", "dd_spec_verify_noalloc", "dd_cache_plan", "dd_cache_append",
    "dd_cache_attention_workspace_bytes", "dd_cache_attention", "dd_logits_edit", "dd_cached_workspace_bytes",
    "dd_denoise_forward_cached", "dd_token_sample", "dd_logits_truncate", "dd_cache_fork_workspace_bytes",
    "dd_cache_fork", "dd_cache_compact_workspace_bytes", "dd_cache_compact", "dd_cache_copy", "dd_profile_begin",
    "dd_profile_end", "dd_profile_num_classes", "dd_profile_read",
]


class DDConfig(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("d_mlp", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("mask_id", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("prior", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("time_cond", ctypes.c_int32), ("norm", ctypes.c_int32), ("norm_eps", ctypes.c_float),
                ("lora_rank", ctypes.c_int32), ("lora_alpha", ctypes.c_float)]


class DDLoopWsLayout(ctypes.Structure):
    _fields_ = [("err", ctypes.c_size_t), ("logits", ctypes.c_size_t), ("rows", ctypes.c_size_t),
                ("count", ctypes.c_size_t), ("glse", ctypes.c_size_t), ("cand", ctypes.c_size_t),
                ("row_lse", ctypes.c_size_t),
                ("logits_ld", ctypes.c_int64), ("glse_ld", ctypes.c_int64)]


class DDCache(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int32), ("block", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class DDCacheMap(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int32), ("T", ctypes.c_int32), ("ld_table", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("held", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("row_start", ctypes.c_void_p), ("row_seq", ctypes.c_void_p), ("row_pos", ctypes.c_void_p),
                ("slots", ctypes.c_void_p)]


class DDLogitsEdits(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("ld_history", ctypes.c_int64), ("hist_len", ctypes.c_void_p),
                ("repetition", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p), ("n_bias", ctypes.c_int32),
                ("allow", ctypes.c_void_p), ("ld_allow", ctypes.c_int64), ("n_allow", ctypes.c_int32),
                ("allow_id", ctypes.c_void_p)]


class DDSampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p)]


class DDError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2609_04010_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        c = ctypes
        P = c.c_void_p
        cfgp = c.POINTER(DDConfig)
        cachep, mapp = c.POINTER(DDCache), c.POINTER(DDCacheMap)
        sig = {
            "dd_param_count": (c.c_int32, [cfgp]),
            "dd_param_tensor": (c.c_int32, [cfgp, c.c_int32, c.POINTER(c.c_size_t),
                                            c.POINTER(c.c_int64), c.POINTER(c.c_int64)]),
            "dd_param_bytes": (c.c_size_t, [cfgp]),
            "dd_workspace_bytes": (c.c_size_t, [cfgp, c.c_int32, c.c_int32]),
            "dd_loop_workspace_bytes": (c.c_size_t, [cfgp, c.c_int32, c.c_int32]),
            "dd_loop_workspace_layout": (c.c_int32, [cfgp, c.c_int32, c.c_int32, c.POINTER(DDLoopWsLayout)]),
            "dd_logits_ld": (c.c_int64, [c.c_int32]),
            "dd_noise_width": (c.c_int32, [c.c_int32, c.c_int32]),
            "dd_status_str": (c.c_char_p, [c.c_int32]),
            "dd_last_error": (c.c_char_p, []),
            "dd_workspace_reset": (c.c_int32, [P, P]),
            "dd_read_device_error": (c.c_int32, [P, c.POINTER(c.c_int32), P]),
            "dd_init_params": (c.c_int32, [cfgp, P, c.c_size_t, c.c_uint64, P, P]),
            "dd_denoise_forward": (c.c_int32, [cfgp, P, P, c.c_int32, c.c_int32, c.c_double, P,
                                               c.c_int64, P, c.c_size_t, P]),
            "dd_attn_mask_build": (c.c_int32, [c.c_int32, c.c_int32, c.c_int32, c.POINTER(c.c_int32)]),
            "dd_denoise_forward_ex": (c.c_int32, [cfgp, P, P, c.c_int32, c.c_int32, c.c_double, P, P,
                                                  P, c.c_int64, P, c.c_size_t, P]),
            "dd_posterior_sample": (c.c_int32, [c.c_int32, P, c.c_int32, c.c_int64, c.c_int32,
                                                c.c_int32, c.c_int32, P, c.c_double, c.c_double, P,
                                                c.c_uint64, c.c_uint32, c.c_uint32, P, P, P, P, P]),
            "dd_psi_posterior_sample": (c.c_int32, [c.c_int32, P, c.c_int32, c.c_int64, c.c_int32,
                                                    c.c_int32, c.c_int32, P, c.c_double, c.c_double,
                                                    c.c_double, P, c.c_uint64, c.c_uint32, c.c_uint32,
                                                    P, P, P, P, P]),
            "dd_sample_loop": (c.c_int32, [cfgp, P, c.c_int32, c.c_int32, c.c_int32,
                                           c.POINTER(c.c_double), P, P, c.c_uint64, P, P,
                                           c.c_size_t, P]),
            "dd_psi_sample_loop": (c.c_int32, [cfgp, P, c.c_int32, c.c_int32, c.c_int32,
                                               c.POINTER(c.c_double), c.POINTER(c.c_double), c.c_uint32,
                                               P, P, c.c_uint64, P, P, c.c_size_t, P]),
            "dd_gaussian_latent_argmax": (c.c_int32, [P, c.c_int32, c.c_int32, c.c_double,
                                                      c.c_double, c.c_uint64, c.c_uint32,
                                                      c.c_uint32, P, P, P]),
            "dd_spec_verify_workspace_bytes": (c.c_size_t, [c.c_int32, c.c_int32]),
            "dd_spec_verify_noise_width": (c.c_int32, [c.c_int32, c.c_int32]),
            "dd_spec_verify": (c.c_int32, [P, P, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int32, P,
                                           P, c.c_uint64, c.c_uint32, c.c_uint32, P, P, P, c.c_size_t, P,
                                           P]),
            "dd_spec_verify_noalloc": (c.c_int32, [P, P, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int32,
                                                   P, P, c.c_uint64, c.c_uint32, c.c_uint32, P, P, P, P]),
            "dd_cache_plan": (c.c_int32, [cachep, mapp, P, P, P, P, P, P, P, P]),
            "dd_cache_append": (c.c_int32, [cachep, P, P, mapp, P, P, c.c_int32, c.c_int64, P, P]),
            "dd_cache_attention_workspace_bytes": (c.c_size_t, [cachep, c.c_int32, c.c_int32, c.c_int32, c.c_int32,
                                                                c.c_int32]),
            "dd_cache_attention": (c.c_int32, [cachep, P, P, mapp, P, c.c_int64, P, c.c_int64, c.c_int32, c.c_int32,
                                               c.c_int32, c.c_double, c.c_int32, c.c_int32, P, c.c_size_t, P, P]),
            "dd_cached_workspace_bytes": (c.c_size_t, [cfgp, cachep, c.c_int32, c.c_int32, c.c_int32, c.c_int32]),
            "dd_denoise_forward_cached": (c.c_int32, [cfgp, P, P, c.c_double, cachep, P, P, mapp, c.c_int32, c.c_int32,
                                                      c.c_int32, P, P, c.c_int64, P, c.c_size_t, P]),
            "dd_logits_edit": (c.c_int32, [P, c.c_int32, c.c_int64, c.c_int32, c.c_int32, P, c.c_int32,
                                           c.POINTER(DDLogitsEdits), P, P]),
            "dd_token_sample": (c.c_int32, [P, c.c_int32, c.c_int64, c.c_int32, c.c_int32, P, c.c_int32, c.c_int32,
                                            c.POINTER(DDSampling), P, c.c_uint64, c.c_uint32, c.c_uint32, P, P, P, P, P]),
            "dd_logits_truncate": (c.c_int32, [P, c.c_int32, c.c_int64, c.c_int32, c.c_int32, P, c.c_int32,
                                               c.POINTER(DDSampling), P, P, P]),
            "dd_cache_fork_workspace_bytes": (c.c_size_t, [cachep, c.c_int32, c.c_int32]),
            "dd_cache_fork": (c.c_int32, [cachep, mapp, mapp, P, P, P, P, P, P, P, P, P, c.c_size_t, P, P]),
            "dd_cache_compact_workspace_bytes": (c.c_size_t, [cachep]),
            "dd_cache_compact": (c.c_int32, [cachep, mapp, P, P, P, P, P, P, c.c_size_t, P, P]),
            "dd_cache_copy": (c.c_int32, [cachep, P, P, c.c_int32, P, P, c.c_int32, P, P]),
            "dd_profile_begin": (c.c_int32, [c.c_int32, c.c_uint32]),
            "dd_profile_end": (c.c_int32, []),
            "dd_profile_num_classes": (c.c_int32, []),
            "dd_profile_read": (c.c_int32, [c.c_int32, c.POINTER(c.c_char_p),
                                            c.POINTER(c.c_int64), c.POINTER(c.c_double)]),
        }
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype = res
            f.argtypes = args
        _lib = L
    return _lib


def _check(st):
    if st != 0:
        raise DDError(st, lib().dd_last_error().decode())


def default_mask_id(prior, V):
    """The mask id a prior takes: V (the K-th category) for the masked prior, -1 for the uniform."""
    return int(V) if prior == "mask" else -1


def make_config(cfg):
    """DDConfig from the architecture dictionary used by the workloads and the oracle."""
    mid = cfg.get("mask_id", default_mask_id(cfg["prior"], cfg["vocab"]))
    return DDConfig(int(cfg["n_layers"]), int(cfg["d_model"]), int(cfg["n_heads"]),
                    int(cfg["d_mlp"]), int(cfg["vocab"]), int(mid), int(cfg["max_len"]),
                    DD_PRIOR_MASK if cfg["prior"] == "mask" else DD_PRIOR_UNIFORM,
                    DD_BF16 if cfg["dtype"] == "bf16" else DD_FP32,
                    1 if cfg.get("time_cond", True) else 0, norm_code(cfg.get("norm", "layer")),
                    float(cfg.get("norm_eps", 1e-5)),
                    int(cfg.get("lora_rank", 0) or 0), float(cfg.get("lora_alpha", 0.0) or 0.0))


def norm_code(norm):
    """dd_norm of a normalisation name: "layer" (LayerNorm) or "rms" (RMSNorm)."""
    if norm not in ("layer", "rms"):
        raise ValueError(f"unknown norm {norm!r}")
    return DD_NORM_RMS if norm == "rms" else DD_NORM_LAYER


def prior_code(prior):
    return DD_PRIOR_MASK if prior == "mask" else DD_PRIOR_UNIFORM


def dtype_code(dtype):
    return DD_BF16 if dtype == "bf16" else DD_FP32


# ---------------------------------------------------------------- host-only queries

def param_count(cfg):
    return lib().dd_param_count(ctypes.byref(make_config(cfg)))


def param_tensor(cfg, tid):
    off, r, c = ctypes.c_size_t(), ctypes.c_int64(), ctypes.c_int64()
    _check(lib().dd_param_tensor(ctypes.byref(make_config(cfg)), tid, ctypes.byref(off),
                                 ctypes.byref(r), ctypes.byref(c)))
    return off.value, r.value, c.value


def param_bytes(cfg):
    return lib().dd_param_bytes(ctypes.byref(make_config(cfg)))


def workspace_bytes(cfg, B, L):
    return lib().dd_workspace_bytes(ctypes.byref(make_config(cfg)), B, L)


def loop_workspace_bytes(cfg, B, L):
    return lib().dd_loop_workspace_bytes(ctypes.byref(make_config(cfg)), B, L)


def loop_workspace_layout(cfg, B, L):
    """dict of the loop workspace regions (byte offsets, row strides) of dd_loop_workspace_layout."""
    out = DDLoopWsLayout()
    _check(lib().dd_loop_workspace_layout(ctypes.byref(make_config(cfg)), int(B), int(L), ctypes.byref(out)))
    return {n: getattr(out, n) for n, _ in DDLoopWsLayout._fields_}


def logits_ld(V):
    return lib().dd_logits_ld(V)


def noise_width(prior, V):
    return lib().dd_noise_width(prior_code(prior), V)


def pack_params(cfg, tensors_by_id):
    """Host blob in the library's parameter layout from a list of float arrays (id order)."""
    nbytes = param_bytes(cfg)
    blob = np.zeros(nbytes, dtype=np.uint8)
    for tid, arr in enumerate(tensors_by_id):
        off, r, c = param_tensor(cfg, tid)
        a = np.asarray(arr, dtype=np.float64).reshape(-1)
        assert a.size == r * c, (tid, a.shape, r, c)
        f = a.astype(np.float32)
        if cfg["dtype"] == "bf16":
            u = f.view(np.uint32)
            if not np.array_equal(u & 0xFFFF, np.zeros_like(u)):
                raise ValueError(f"tensor {tid} is not exactly representable in bf16")
            raw = (u >> 16).astype(np.uint16).view(np.uint8)
        else:
            raw = f.view(np.uint8)
        blob[off:off + raw.size] = raw
    return blob


# ---------------------------------------------------------------- device calls

def _torch():
    import torch
    return torch


def _stream():
    return ctypes.c_void_p(_torch().cuda.current_stream().cuda_stream)


def _ptr(t, nbytes, name, dtype=None):
    """Device pointer of a contiguous GPU tensor holding at least `nbytes` bytes."""
    if t is None:
        return None
    torch = _torch()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise ValueError(f"{name} holds {have} bytes, needs {nbytes}")
    return ctypes.c_void_p(t.data_ptr())


def init_params(cfg, params, seed=0, host_blob=None):
    need = param_bytes(cfg)
    src = None
    if host_blob is not None:
        host_blob = np.ascontiguousarray(host_blob, dtype=np.uint8)
        if host_blob.size < need:
            raise ValueError("host blob too small")
        src = host_blob.ctypes.data_as(ctypes.c_void_p)
    _check(lib().dd_init_params(ctypes.byref(make_config(cfg)), _ptr(params, need, "params"),
                                params.numel() * params.element_size(), int(seed), src, _stream()))
    if host_blob is not None:
        _torch().cuda.current_stream().synchronize()   # the host blob must outlive the copy


def denoise_forward(cfg, params, z_t, B, L, alpha_t, logits, ld, ws):
    torch = _torch()
    es = 2 if cfg["dtype"] == "bf16" else 4
    M = B * L
    _check(lib().dd_denoise_forward(
        ctypes.byref(make_config(cfg)), _ptr(params, param_bytes(cfg), "params"),
        _ptr(z_t, 4 * M, "z_t", torch.int32), B, L, float(alpha_t),
        _ptr(logits, es * M * ld, "logits"), int(ld),
        _ptr(ws, workspace_bytes(cfg, B, L), "ws"), ws.numel() * ws.element_size(), _stream()))


def attn_mask_build(pattern, L, block=0):
    """Host int32 array [3, L] (pre, lo, hi) of a named pattern (see ATTN_PATTERNS)."""
    out = np.zeros(3 * L, dtype=np.int32)
    code = ATTN_PATTERNS[pattern] if isinstance(pattern, str) else int(pattern)
    _check(lib().dd_attn_mask_build(code, int(L), int(block),
                                    out.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))))
    return out.reshape(3, L)


def denoise_forward_ex(cfg, params, z_t, B, L, alpha_t, logits, ld, ws, attn_mask=None, lora_gate=None):
    """dd_denoise_forward_ex; attn_mask is a device int32 tensor of 3 L entries, lora_gate of L."""
    torch = _torch()
    es = 2 if cfg["dtype"] == "bf16" else 4
    M = B * L
    _check(lib().dd_denoise_forward_ex(
        ctypes.byref(make_config(cfg)), _ptr(params, param_bytes(cfg), "params"),
        _ptr(z_t, 4 * M, "z_t", torch.int32), B, L, float(alpha_t),
        _ptr(attn_mask, 12 * L, "attn_mask", torch.int32) if attn_mask is not None else None,
        _ptr(lora_gate, 4 * L, "lora_gate", torch.int32) if lora_gate is not None else None,
        _ptr(logits, es * M * ld, "logits"), int(ld),
        _ptr(ws, workspace_bytes(cfg, B, L), "ws"), ws.numel() * ws.element_size(), _stream()))


def _posterior_args(prior, logits, logits_dtype, ld, rows, V, z_t, noise_words, z_s, row_lse, probs,
                    dev_err):
    torch = _torch()
    es = 2 if logits_dtype == "bf16" else 4
    K = V + 1 if prior == "mask" else V
    nu = noise_width(prior, V)
    lg = _ptr(logits, es * rows * ld, "logits") if rows > 0 else None
    return (lg, _ptr(z_t, 4 * rows, "z_t", torch.int32),
            _ptr(noise_words, 4 * rows * nu, "noise_words", torch.int32) if noise_words is not None else None,
            _ptr(z_s, 4 * rows, "z_s", torch.int32),
            _ptr(row_lse, 4 * rows, "row_lse", torch.float32) if row_lse is not None else None,
            _ptr(probs, 4 * rows * K, "probs", torch.float32) if probs is not None else None,
            _ptr(dev_err, 4, "dev_err", torch.int32) if dev_err is not None else None)


def posterior_sample(prior, logits, logits_dtype, ld, rows, V, z_t, alpha_t, alpha_s, z_s,
                     noise_words=None, seed=0, step=0, row0=0, probs=None, dev_err=None, row_lse=None,
                     mask_id=None):
    """dd_posterior_sample; mask_id defaults to the prior's (V for "mask", -1 for "uniform")."""
    lg, zt, nw, zs, rl, pr, er = _posterior_args(prior, logits, logits_dtype, ld, rows, V, z_t, noise_words,
                                                 z_s, row_lse, probs, dev_err)
    mid = default_mask_id(prior, V) if mask_id is None else int(mask_id)
    _check(lib().dd_posterior_sample(
        prior_code(prior), lg, dtype_code(logits_dtype), int(ld), int(rows), int(V), mid, zt, float(alpha_t),
        float(alpha_s), nw, int(seed) & 0xFFFFFFFFFFFFFFFF, int(step), int(row0), zs, rl, pr, er, _stream()))


def psi_posterior_sample(prior, logits, logits_dtype, ld, rows, V, z_t, alpha_t, alpha_s, kappa, z_s,
                         noise_words=None, seed=0, step=0, row0=0, probs=None, dev_err=None, row_lse=None,
                         mask_id=None):
    lg, zt, nw, zs, rl, pr, er = _posterior_args(prior, logits, logits_dtype, ld, rows, V, z_t, noise_words,
                                                 z_s, row_lse, probs, dev_err)
    mid = default_mask_id(prior, V) if mask_id is None else int(mask_id)
    _check(lib().dd_psi_posterior_sample(
        prior_code(prior), lg, dtype_code(logits_dtype), int(ld), int(rows), int(V), mid, zt, float(alpha_t),
        float(alpha_s), float(kappa), nw, int(seed) & 0xFFFFFFFFFFFFFFFF, int(step), int(row0), zs, rl, pr, er,
        _stream()))


def sample_loop(cfg, params, B, L, T, alphas, z, ws, noise_words=None, noise_seed=0, z_trace=None,
                kappas=None, posterior_pass=False, store_free=False):
    """dd_sample_loop, or dd_psi_sample_loop when kappas (T + 1 values) is given or a flag is set:
    posterior_pass (DD_LOOP_POSTERIOR_PASS), store_free (DD_LOOP_STORE_FREE)."""
    torch = _torch()
    M = B * L
    a = np.ascontiguousarray(alphas, dtype=np.float64)
    if a.shape != (T + 1,):
        raise ValueError("alphas must hold T + 1 values")
    nu = noise_width(cfg["prior"], cfg["vocab"])
    dp = ctypes.POINTER(ctypes.c_double)
    head = (ctypes.byref(make_config(cfg)), _ptr(params, param_bytes(cfg), "params"), B, L, T, a.ctypes.data_as(dp))
    tail = (_ptr(z, 4 * M, "z", torch.int32),
            _ptr(noise_words, 4 * T * M * nu, "noise_words", torch.int32) if noise_words is not None else None,
            int(noise_seed) & 0xFFFFFFFFFFFFFFFF,
            _ptr(z_trace, 4 * (T + 1) * M, "z_trace", torch.int32) if z_trace is not None else None,
            _ptr(ws, loop_workspace_bytes(cfg, B, L), "ws"), ws.numel() * ws.element_size(), _stream())
    if kappas is None and not posterior_pass and not store_free:
        _check(lib().dd_sample_loop(*head, *tail))
    else:
        k = None
        if kappas is not None:
            k = np.ascontiguousarray(kappas, dtype=np.float64)
            if k.shape != (T + 1,):
                raise ValueError("kappas must hold T + 1 values")
        flags = (DD_LOOP_POSTERIOR_PASS if posterior_pass else 0) | (DD_LOOP_STORE_FREE if store_free else 0)
        _check(lib().dd_psi_sample_loop(*head, k.ctypes.data_as(dp) if k is not None else None, flags, *tail))


def spec_verify_workspace_bytes(S, B):
    return int(lib().dd_spec_verify_workspace_bytes(int(S), int(B)))


def spec_verify_noise_width(B, V):
    return int(lib().dd_spec_verify_noise_width(int(B), int(V)))


def spec_verify(p_logits, q_logits, logits_dtype, ld, S, B, V, draft, n_out, z_out, ws, noise_words=None,
                seed=0, step=0, row0=0, dev_err=None):
    torch = _torch()
    es = 2 if logits_dtype == "bf16" else 4
    nu = spec_verify_noise_width(B, V)
    _check(lib().dd_spec_verify(
        _ptr(p_logits, es * S * B * ld, "p_logits"),
        _ptr(q_logits, es * S * (B - 1) * ld, "q_logits") if B > 1 else None, dtype_code(logits_dtype),
        int(ld), int(S), int(B), int(V),
        _ptr(draft, 4 * S * (B - 1), "draft", torch.int32) if B > 1 else None,
        _ptr(noise_words, 4 * S * nu, "noise_words", torch.int32) if noise_words is not None else None,
        int(seed) & 0xFFFFFFFFFFFFFFFF, int(step), int(row0), _ptr(n_out, 4 * S, "n_out", torch.int32),
        _ptr(z_out, 4 * S, "z_out", torch.int32), _ptr(ws, spec_verify_workspace_bytes(S, B), "ws"),
        ws.numel() * ws.element_size(), _ptr(dev_err, 4, "dev_err", torch.int32) if dev_err is not None else None,
        _stream()))


SPEC_VERIFY_NOALLOC_ROWS = 1 << 18


def spec_verify_noalloc(p_logits, q_logits, logits_dtype, ld, S, B, V, draft, n_out, z_out, noise_words=None,
                        seed=0, step=0, row0=0, dev_err=None):
    """dd_spec_verify_noalloc: dd_spec_verify without a workspace (library-held device array)."""
    torch = _torch()
    es = 2 if logits_dtype == "bf16" else 4
    nu = spec_verify_noise_width(B, V)
    _check(lib().dd_spec_verify_noalloc(
        _ptr(p_logits, es * S * B * ld, "p_logits"),
        _ptr(q_logits, es * S * (B - 1) * ld, "q_logits") if B > 1 else None, dtype_code(logits_dtype),
        int(ld), int(S), int(B), int(V),
        _ptr(draft, 4 * S * (B - 1), "draft", torch.int32) if B > 1 else None,
        _ptr(noise_words, 4 * S * nu, "noise_words", torch.int32) if noise_words is not None else None,
        int(seed) & 0xFFFFFFFFFFFFFFFF, int(step), int(row0), _ptr(n_out, 4 * S, "n_out", torch.int32),
        _ptr(z_out, 4 * S, "z_out", torch.int32),
        _ptr(dev_err, 4, "dev_err", torch.int32) if dev_err is not None else None, _stream()))


def gaussian_latent_argmax(x, rows, V, alpha_tilde, sigma, seed, step, z_out, row0=0, dev_err=None):
    torch = _torch()
    _check(lib().dd_gaussian_latent_argmax(
        _ptr(x, 4 * rows, "x", torch.int32), int(rows), int(V), float(alpha_tilde), float(sigma),
        int(seed) & 0xFFFFFFFFFFFFFFFF, int(step), int(row0), _ptr(z_out, 4 * rows, "z_out", torch.int32),
        _ptr(dev_err, 4, "dev_err", torch.int32) if dev_err is not None else None, _stream()))


# ---------------------------------------------------------------- cached context

# These calls are short on the GPU, so what a wrapper costs on the host is most of a small one: the current
# device and its stream are looked up once per call, and each tensor in as few calls as the checks need.

_here, _raw_stream = None, None


def _current():
    """(index, stream) of the current GPU."""
    global _here, _raw_stream
    if _here is None:
        torch = _torch()
        torch.cuda.init()
        _here = torch.cuda.current_device
        # torch's own accessor without the Stream object around it, where this torch has it
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda dev: torch.cuda.current_stream(dev).cuda_stream)
    dev = _here()
    return dev, _raw_stream(dev)


def _other_device(t, dev, name):
    raise ValueError(f"{name} must be on the current GPU (cuda:{dev}), got {t.device}")


def _dev(t, dev, n, name, dtype):
    """Device pointer of a contiguous tensor of at least n entries of `dtype` on GPU `dev` (None for None)."""
    if t is None:
        return None
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        _other_device(t, dev, name)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < n:
        raise ValueError(f"{name} holds {t.numel()} entries, needs {n}")
    return t.data_ptr()


def _rows(t, dev, n, width, name, dtype):
    """(device pointer, row stride) of a tensor [n or more][width or more] with neighbouring columns: a view of
    columns of wider rows will do."""
    if t.dtype is not dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        _other_device(t, dev, name)
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, got {tuple(t.shape)}")
    rows, cols = t.shape
    ld, unit = t.stride()
    if rows < n or cols < width or (unit != 1 and cols > 1) or (rows > 1 and ld < width):
        raise ValueError(f"{name} must be [{n}, {width}] with neighbouring columns and rows that do not overlap, got "
                         f"{(rows, cols)} with strides {(ld, unit)}")
    if rows <= 1:      # the stride of a single row says nothing
        unit = 16 // t.element_size()
        ld = (width + unit - 1) // unit * unit
    return t.data_ptr(), ld


def _float_code(t, name):
    torch = _torch()
    if t.dtype is torch.bfloat16:
        return DD_BF16
    if t.dtype is torch.float32:
        return DD_FP32
    raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")


def cache_config(n_blocks, block, n_kv_heads, head_dim):
    """dd_cache of a pool: n_blocks blocks of `block` tokens, n_kv_heads heads of head_dim numbers."""
    return DDCache(int(n_blocks), int(block), int(n_kv_heads), int(head_dim))


def cache_tensors(cc, layers=None, device="cuda"):
    """(codes, scales) of one layer, uint8 [n_blocks, heads, 2 block dh] and fp32 [n_blocks, heads, 2], or of
    `layers` of them in front; zeroed."""
    torch = _torch()
    lead = (cc.n_blocks, cc.n_kv_heads) if layers is None else (layers, cc.n_blocks, cc.n_kv_heads)
    return (torch.zeros((*lead, 2 * cc.block * cc.head_dim), dtype=torch.uint8, device=device),
            torch.zeros((*lead, 2), dtype=torch.float32, device=device))


class CacheMap:
    """dd_cache_map over int32 tensors block_table [S, ld_table], held [S], kv_len [S], row_start [S + 1],
    row_seq, row_pos and slots [T], which it keeps."""

    def __init__(self, block_table, held, kv_len, row_start, row_seq, row_pos, slots):
        i32 = _torch().int32
        if block_table.dim() != 2:
            raise ValueError("block_table must be [S, ld_table]")
        if block_table.get_device() < 0:
            raise ValueError(f"block_table must be on the GPU, got {block_table.device}")
        S, ld = block_table.shape
        T = row_seq.numel()
        self.block_table, self.held, self.kv_len, self.row_start = block_table, held, kv_len, row_start
        self.row_seq, self.row_pos, self.slots = row_seq, row_pos, slots
        self.S, self.T, self.ld_table = S, T, ld
        self.device = dev = block_table.get_device()
        self.struct = DDCacheMap(S, T, ld, _dev(block_table, dev, S * ld, "block_table", i32), _dev(held, dev, S, "held", i32),
                                 _dev(kv_len, dev, S, "kv_len", i32), _dev(row_start, dev, S + 1, "row_start", i32),
                                 _dev(row_seq, dev, T, "row_seq", i32), _dev(row_pos, dev, T, "row_pos", i32),
                                 _dev(slots, dev, T, "slots", i32))
        self.ref = ctypes.byref(self.struct)

    def on(self, dev):
        """The struct's reference, for calls on GPU `dev`."""
        if self.device != dev:
            raise ValueError(f"the map must be on the current GPU (cuda:{dev}), got cuda:{self.device}")
        return self.ref

    @classmethod
    def empty(cls, S, T, ld_table, device="cuda"):
        """A map of S sequences, T rows and tables of ld_table entries that hold no block yet."""
        torch = _torch()
        z = lambda *n: torch.zeros(n, dtype=torch.int32, device=device)   # noqa: E731
        return cls(z(S, ld_table).fill_(-1), z(S), z(S), z(S + 1), z(T), z(T), z(T))


def cache_plan(cc, m, seq_len, n_new, held, free_blocks, n_free, n_free_out, dev_err=None):
    i32, S = _torch().int32, m.S
    dev, stream = _current()
    _check(lib().dd_cache_plan(
        ctypes.byref(cc), m.on(dev), _dev(seq_len, dev, S, "seq_len", i32), _dev(n_new, dev, S, "n_new", i32),
        _dev(held, dev, S, "held", i32), _dev(free_blocks, dev, cc.n_blocks, "free_blocks", i32),
        _dev(n_free, dev, 1, "n_free", i32), _dev(n_free_out, dev, 1, "n_free_out", i32),
        _dev(dev_err, dev, 1, "dev_err", i32), stream))


def _cache_ptrs(cc, dev, codes, scales, layers=1):
    torch = _torch()
    n = layers * cc.n_blocks * cc.n_kv_heads * 2
    t = torch.uint8 if codes.dtype is not torch.float8_e4m3fn else torch.float8_e4m3fn
    return (_dev(codes, dev, n * cc.block * cc.head_dim, "codes", t), _dev(scales, dev, n, "scales", torch.float32))


def cache_append(cc, codes, scales, m, k, v, dev_err=None):
    """dd_cache_append; k and v are [T, n_kv_heads head_dim], of one type and row stride (views of packed rows)."""
    dev, stream = _current()
    T, w, t = m.T, cc.n_kv_heads * cc.head_dim, k.dtype
    pk, ld = _rows(k, dev, T, w, "k", t)
    pv, ldv = _rows(v, dev, T, w, "v", t)
    if ld != ldv:
        raise ValueError(f"k and v must have one row stride, got {ld} and {ldv}")
    pc, ps = _cache_ptrs(cc, dev, codes, scales)
    _check(lib().dd_cache_append(ctypes.byref(cc), pc, ps, m.on(dev), pk, pv, _float_code(k, "k"), ld,
                                 _dev(dev_err, dev, 1, "dev_err", _torch().int32), stream))


def cache_attention_workspace_bytes(cc, S, T, n_heads, max_new, max_kv):
    return int(lib().dd_cache_attention_workspace_bytes(ctypes.byref(cc), int(S), int(T), int(n_heads), int(max_new),
                                                        int(max_kv)))


def cache_attention(cc, codes, scales, m, q, out, n_heads, max_new, max_kv, ws=None, pattern="causal",
                    softmax_scale=None, dev_err=None):
    """dd_cache_attention; q and out are [T, n_heads head_dim]; softmax_scale defaults to head_dim ** -0.5."""
    dev, stream = _current()
    T, w, t = m.T, n_heads * cc.head_dim, q.dtype
    pq, ldq = _rows(q, dev, T, w, "q", t)
    po, ldo = _rows(out, dev, T, w, "out", t)
    pc, ps = _cache_ptrs(cc, dev, codes, scales)
    pw, wb = (None, 0) if ws is None else (_dev(ws, dev, 0, "ws", ws.dtype), ws.numel() * ws.element_size())
    _check(lib().dd_cache_attention(
        ctypes.byref(cc), pc, ps, m.on(dev), pq, ldq, po, ldo, _float_code(q, "q"), n_heads, ATTN_PATTERNS[pattern],
        softmax_scale if softmax_scale is not None else cc.head_dim ** -0.5, max_new, max_kv, pw, wb,
        _dev(dev_err, dev, 1, "dev_err", _torch().int32), stream))


def cached_workspace_bytes(cfg, cc, S, T, max_new, max_kv):
    return int(lib().dd_cached_workspace_bytes(ctypes.byref(make_config(cfg)), ctypes.byref(cc), int(S), int(T),
                                               int(max_new), int(max_kv)))


def denoise_forward_cached(cfg, params, z_t, alpha_t, cc, codes, scales, m, logits, ld, ws, max_new, max_kv,
                           pattern="causal", lora_gate=None):
    """dd_denoise_forward_cached; codes and scales hold the caches of the n_layers layers (cache_tensors with
    layers=n_layers)."""
    torch = _torch()
    i32 = torch.int32
    dev, stream = _current()
    pc, ps = _cache_ptrs(cc, dev, codes, scales, cfg["n_layers"])
    pw = _dev(ws, dev, 0, "ws", ws.dtype)
    _check(lib().dd_denoise_forward_cached(
        ctypes.byref(make_config(cfg)), _ptr(params, param_bytes(cfg), "params"), _dev(z_t, dev, m.T, "z_t", i32),
        float(alpha_t), ctypes.byref(cc), pc, ps, m.on(dev), ATTN_PATTERNS[pattern], max_new, max_kv,
        _dev(lora_gate, dev, m.T, "lora_gate", i32),
        _dev(logits, dev, m.T * ld, "logits", torch.bfloat16 if cfg["dtype"] == "bf16" else torch.float32), ld,
        pw, ws.numel() * ws.element_size(), stream))


def logits_edit(logits, logits_dtype, ld, rows, V, out, rows_per_seq=1, history=None, hist_len=None, repetition=None,
                presence=None, frequency=None, bias_ids=None, bias_values=None, allow=None, allow_id=None, dev_err=None):
    """dd_logits_edit; history [n_seq, entries], bias_ids / bias_values [n_seq, n_bias] and allow [n_allow, words]
    give their sizes by their shapes (int32, or int32 holding the masks' bits)."""
    torch = _torch()
    i32, f32 = torch.int32, torch.float32
    t = torch.bfloat16 if logits_dtype == "bf16" else f32
    dev, stream = _current()
    n_seq = -(-rows // rows_per_seq) if rows_per_seq > 0 else 0
    lh = nb = na = la = 0
    if history is not None:
        _two_dims(history, "history")
        lh = history.shape[1]
    if bias_ids is not None:
        _two_dims(bias_ids, "bias_ids")
        nb = bias_ids.shape[1]
        if bias_values is None or bias_values.shape != bias_ids.shape:
            raise ValueError("bias_values must have the shape of bias_ids")
    if allow is not None:
        _two_dims(allow, "allow")
        na, la = allow.shape
    e = DDLogitsEdits(
        _dev(history, dev, n_seq * lh, "history", i32), lh, _dev(hist_len, dev, rows, "hist_len", i32),
        _dev(repetition, dev, n_seq, "repetition", f32), _dev(presence, dev, n_seq, "presence", f32),
        _dev(frequency, dev, n_seq, "frequency", f32), _dev(bias_ids, dev, n_seq * nb, "bias_ids", i32),
        _dev(bias_values, dev, n_seq * nb, "bias_values", f32), nb, _dev(allow, dev, na * la, "allow", i32), la, na,
        _dev(allow_id, dev, rows, "allow_id", i32))
    _check(lib().dd_logits_edit(
        _dev(logits, dev, rows * ld, "logits", t), dtype_code(logits_dtype), ld, rows, V, _dev(out, dev, rows * ld, "out", t),
        rows_per_seq, ctypes.byref(e), _dev(dev_err, dev, 1, "dev_err", i32), stream))


def _sampling(dev, entries, temperature, top_k, top_p, min_p):
    torch = _torch()
    f32 = torch.float32
    return DDSampling(_dev(temperature, dev, entries, "temperature", f32), _dev(top_k, dev, entries, "top_k", torch.int32),
                      _dev(top_p, dev, entries, "top_p", f32), _dev(min_p, dev, entries, "min_p", f32))


def token_sample(logits, logits_dtype, ld, rows, V, z_out, n, row_ids=None, draws_per_seq=1, temperature=None, top_k=None,
                 top_p=None, min_p=None, noise_words=None, seed=0, step=0, row0=0, logp=None, n_kept=None, dev_err=None):
    """dd_token_sample: n draws, draw i from row row_ids[i] (or i) under the settings of entry i // draws_per_seq."""
    torch = _torch()
    i32 = torch.int32
    dev, stream = _current()
    how = _sampling(dev, -(-n // draws_per_seq) if draws_per_seq > 0 else 0, temperature, top_k, top_p, min_p)
    _check(lib().dd_token_sample(
        _dev(logits, dev, rows * ld, "logits", torch.bfloat16 if logits_dtype == "bf16" else torch.float32),
        dtype_code(logits_dtype), ld, rows, V, _dev(row_ids, dev, n, "row_ids", i32), n, draws_per_seq, ctypes.byref(how),
        _dev(noise_words, dev, n, "noise_words", i32), seed & 0xFFFFFFFFFFFFFFFF, step, row0, _dev(z_out, dev, n, "z_out", i32),
        _dev(logp, dev, n, "logp", torch.float32), _dev(n_kept, dev, n, "n_kept", i32), _dev(dev_err, dev, 1, "dev_err", i32),
        stream))


def logits_truncate(logits, logits_dtype, ld, rows, V, out, rows_per_seq=1, temperature=None, top_k=None, top_p=None,
                    min_p=None, n_kept=None, dev_err=None):
    """dd_logits_truncate; row m takes the settings of entry m // rows_per_seq."""
    torch = _torch()
    i32 = torch.int32
    t = torch.bfloat16 if logits_dtype == "bf16" else torch.float32
    dev, stream = _current()
    how = _sampling(dev, -(-rows // rows_per_seq) if rows_per_seq > 0 else 0, temperature, top_k, top_p, min_p)
    _check(lib().dd_logits_truncate(
        _dev(logits, dev, rows * ld, "logits", t), dtype_code(logits_dtype), ld, rows, V, _dev(out, dev, rows * ld, "out", t),
        rows_per_seq, ctypes.byref(how), _dev(n_kept, dev, rows, "n_kept", i32), _dev(dev_err, dev, 1, "dev_err", i32), stream))


def cache_fork_workspace_bytes(cc, S, S_to):
    return int(lib().dd_cache_fork_workspace_bytes(ctypes.byref(cc), int(S), int(S_to)))


def cache_fork(cc, m, to, seq_len, src, free_blocks, n_free, n_free_out, moves, n_moves, ws, keep=None, dev_err=None):
    """dd_cache_fork: the sequences of the CacheMap `to` from those of `m`; moves is [to.S, 2]."""
    i32 = _torch().int32
    dev, stream = _current()
    _check(lib().dd_cache_fork(
        ctypes.byref(cc), m.on(dev), to.on(dev), _dev(seq_len, dev, m.S, "seq_len", i32), _dev(src, dev, to.S, "src", i32),
        _dev(keep, dev, to.S, "keep", i32), _dev(free_blocks, dev, cc.n_blocks, "free_blocks", i32),
        _dev(n_free, dev, 1, "n_free", i32), _dev(n_free_out, dev, 1, "n_free_out", i32), _dev(moves, dev, 2 * to.S, "moves", i32),
        _dev(n_moves, dev, 1, "n_moves", i32), _dev(ws, dev, 0, "ws", ws.dtype), ws.numel() * ws.element_size(),
        _dev(dev_err, dev, 1, "dev_err", i32), stream))


def cache_compact_workspace_bytes(cc):
    return int(lib().dd_cache_compact_workspace_bytes(ctypes.byref(cc)))


def cache_compact(cc, m, block_table_out, free_blocks, n_free_out, moves, n_moves, ws, dev_err=None):
    """dd_cache_compact; block_table_out may be m.block_table, moves is [n_blocks // 2 or more, 2]."""
    i32 = _torch().int32
    dev, stream = _current()
    _check(lib().dd_cache_compact(
        ctypes.byref(cc), m.on(dev), _dev(block_table_out, dev, m.S * m.ld_table, "block_table_out", i32),
        _dev(free_blocks, dev, cc.n_blocks, "free_blocks", i32), _dev(n_free_out, dev, 1, "n_free_out", i32),
        _dev(moves, dev, cc.n_blocks // 2 * 2, "moves", i32), _dev(n_moves, dev, 1, "n_moves", i32), _dev(ws, dev, 0, "ws", ws.dtype),
        ws.numel() * ws.element_size(), _dev(dev_err, dev, 1, "dev_err", i32), stream))


def cache_copy(cc, codes, scales, moves, n_moves, layers=1, dev_err=None):
    """dd_cache_copy over the caches of `layers` layers; moves is [max_moves, 2]."""
    i32 = _torch().int32
    dev, stream = _current()
    _two_dims(moves, "moves")
    if moves.shape[1] != 2:
        raise ValueError(f"moves must be [max_moves, 2], got {tuple(moves.shape)}")
    pc, ps = _cache_ptrs(cc, dev, codes, scales, layers)
    _check(lib().dd_cache_copy(ctypes.byref(cc), pc, ps, layers, _dev(moves, dev, 0, "moves", i32),
                               _dev(n_moves, dev, 1, "n_moves", i32), moves.shape[0], _dev(dev_err, dev, 1, "dev_err", i32), stream))


def _two_dims(t, name):
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions, got {tuple(t.shape)}")


def workspace_reset(ws):
    _check(lib().dd_workspace_reset(_ptr(ws, 4, "ws"), _stream()))


def read_device_error(err):
    code = ctypes.c_int32(0)
    st = lib().dd_read_device_error(_ptr(err, 4, "err"), ctypes.byref(code), _stream())
    if st not in (0, 7):
        _check(st)
    return code.value


PROFILE_CLASSES = ["time_embedding", "embed_layernorm", "layernorm", "gemm_qkv", "attention",
                   "gemm_attn_out", "gemm_mlp_up", "gemm_mlp_down", "gemm_vocab",
                   "posterior_sample", "gaussian_latent", "init_params", "copy", "compact_masked",
                   "gemm_lora_down", "cache_plan", "cache_append", "cache_attention", "logits_edit",
                   "token_sample", "logits_truncate", "cache_fork", "cache_copy", "cache_compact"]


def profile_begin(max_launches, classes=None):
    """Start event timing; `classes` is a list of class names (None: every class)."""
    mask = 0
    for name in classes or []:
        mask |= 1 << PROFILE_CLASSES.index(name)
    _check(lib().dd_profile_begin(int(max_launches), mask))


def profile_end():
    _check(lib().dd_profile_end())


def profile_read():
    """{class name: (launches, total ms)} for every class with at least one launch."""
    out = {}
    for c in range(lib().dd_profile_num_classes()):
        name, n, ms = ctypes.c_char_p(), ctypes.c_int64(), ctypes.c_double()
        _check(lib().dd_profile_read(c, ctypes.byref(name), ctypes.byref(n), ctypes.byref(ms)))
        if n.value:
            out[name.value.decode()] = (n.value, ms.value)
    return out
