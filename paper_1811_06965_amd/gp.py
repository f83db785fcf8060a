"""ctypes binding of the partition's C ABI (include/gp.h).

Argument marshalling only: every step of the partition's work runs in the HIP
kernels of libgp.so.  Device buffers are passed as integer device addresses
(e.g. ``tensor.data_ptr()``) and streams as raw HIP stream handles (e.g.
``torch.cuda.current_stream().cuda_stream``).  If the library has not been
built the import-time loader raises: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libgp.so")

GP_OK, GP_ERR_INVALID_ARG, GP_ERR_STATE, GP_ERR_OOM, GP_ERR_HIP, GP_ERR_NONFINITE, GP_ERR_UNSUPPORTED = range(7)
STATUS_NAMES = {0: "GP_OK", 1: "GP_ERR_INVALID_ARG", 2: "GP_ERR_STATE", 3: "GP_ERR_OOM", 4: "GP_ERR_HIP",
                5: "GP_ERR_NONFINITE", 6: "GP_ERR_UNSUPPORTED"}
GP_F32, GP_BF16 = 0, 1
GP_ENCODER, GP_DECODER_CROSS = 0, 1
GP_LOSS_NONE, GP_LOSS_MSE, GP_LOSS_XENT_LS = 0, 1, 2
GP_OPT_SGD, GP_OPT_RMSPROP, GP_OPT_ADAMW = 0, 1, 2

PARAM_IDS = ["ln1_g", "ln1_b", "wq", "bq", "wk", "bk", "wv", "bv", "wo", "bo", "ln2_g", "ln2_b",
             "w1", "b1", "w2", "b2", "xwq", "xbq", "xwk", "xbk", "xwv", "xbv", "xwo", "xbo",
             "ln3_g", "ln3_b", "lnf_g", "lnf_b", "wout", "bout"]
PARAM_ID = {name: i for i, name in enumerate(PARAM_IDS)}

# gp_kernel_role: launch roles of the timers
KERNEL_ROLES = ["none", "qkv.fwd", "qkv.dx", "qkv.dw", "o.fwd", "o.dx", "o.dw", "ffn1.fwd", "ffn1.dx", "ffn1.dw",
                "ffn2.fwd", "ffn2.dx", "ffn2.dw", "xq.fwd", "xq.dx", "xq.dw", "xkv.fwd", "xkv.dx", "xkv.dw",
                "xo.fwd", "xo.dx", "xo.dw", "head.fwd", "head.dx", "head.dw", "attn.fwd", "attn.bwd",
                "xattn.fwd", "xattn.bwd", "ln.fwd", "ln.bwd"]
KERNEL_ROLE = {name: i for i, name in enumerate(KERNEL_ROLES)}
GP_K_NONE, GP_K_COUNT = 0, len(KERNEL_ROLES)

EXPORTS = ["gp_partition_create", "gp_partition_configure", "gp_partition_destroy", "gp_set_param",
           "gp_get_param", "gp_get_grad", "gp_partition_memory", "gp_param_count", "gp_forward_microbatch",
           "gp_backward_microbatch_remat", "gp_accumulate_and_step", "gp_timer_select", "gp_timer_read",
           "gp_timer_reset", "gp_timer_sample", "gp_mfma_peak", "gp_recomputed_output", "gp_memory_plan",
           "gp_forward_microbatch_noalloc", "gp_plan_cells", "gp_stream_create", "gp_stream_destroy",
           "gp_token_logprobs", "gp_token_logprobs_workspace", "gp_token_logprobs_backward", "gp_grad_norm",
           "gp_grad_norm_workspace", "gp_adamw_step", "gp_get_grad_norm", "gp_score_sequences",
           "gp_backward_microbatch_weighted", "gp_get_moment", "gp_set_moment", "gp_get_updates", "gp_set_updates",
           "gp_attention", "gp_attention_workspace", "gp_attention_backward", "gp_relative_buckets", "gp_distill",
           "gp_distill_workspace", "gp_distill_backward", "gp_last_error"]

GP_TOP_MAX, GP_NO_TOKEN, GP_STATE_BLOCK = 32, -1, 256
GP_BUCKETS_MAX, GP_DISTANCE_MAX, GP_DISTILL_MAX = 1024, 1024, 256


class gp_config(ctypes.Structure):
    _fields_ = [("seq_len", ctypes.c_int), ("seqs_per_microbatch", ctypes.c_int),
                ("num_microbatches", ctypes.c_int), ("dtype", ctypes.c_int), ("kind", ctypes.c_int),
                ("mem_seq_len", ctypes.c_int), ("loss", ctypes.c_int), ("vocab", ctypes.c_int),
                ("label_smoothing", ctypes.c_float), ("ln_eps", ctypes.c_float),
                ("check_finite", ctypes.c_int), ("keep_activations", ctypes.c_int), ("optimizer", ctypes.c_int),
                ("rms_decay", ctypes.c_float), ("rms_eps", ctypes.c_float), ("logit_clip", ctypes.c_float),
                ("adam_beta1", ctypes.c_float), ("adam_beta2", ctypes.c_float), ("adam_eps", ctypes.c_float),
                ("weight_decay", ctypes.c_float), ("max_grad_norm", ctypes.c_float)]


class gp_grad_tensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("count", ctypes.c_longlong)]


class gp_adamw_tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("copy", ctypes.c_void_p), ("count", ctypes.c_longlong), ("weight_decay", ctypes.c_double)]


class gp_adamw_config(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int), ("state_bits", ctypes.c_int),
                ("seed", ctypes.c_uint), ("lr", ctypes.c_double), ("beta1", ctypes.c_double),
                ("beta2", ctypes.c_double), ("eps", ctypes.c_double)]


class gp_head_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("seq_stride", ctypes.c_long), ("row_stride", ctypes.c_long),
                ("head_stride", ctypes.c_long)]


class gp_attention_config(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("batch", ctypes.c_int), ("heads", ctypes.c_int), ("kv_heads", ctypes.c_int),
                ("q_len", ctypes.c_int), ("k_len", ctypes.c_int), ("head_dim", ctypes.c_int), ("causal", ctypes.c_int),
                ("scale", ctypes.c_float), ("q_lens", ctypes.c_void_p), ("k_lens", ctypes.c_void_p),
                ("q_starts", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("bucket_of", ctypes.c_void_p),
                ("buckets", ctypes.c_int), ("max_distance", ctypes.c_int)]


class GpError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


_lib = None


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libgp.so (once).  Raises if it is missing: build it first."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build the HIP library first (python -m paper_1811_06965_amd.build)")
    lib = ctypes.CDLL(path)
    P, VP, I, SZ = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    FP = ctypes.POINTER(ctypes.c_float)
    lib.gp_partition_create.argtypes = [I, I, I, I, ctypes.POINTER(P)]
    lib.gp_partition_configure.argtypes = [P, ctypes.POINTER(gp_config)]
    lib.gp_partition_destroy.argtypes = [P]
    for f in (lib.gp_set_param, lib.gp_get_param, lib.gp_get_grad):
        f.argtypes = [P, I, I, FP, SZ]
    for f in (lib.gp_get_moment, lib.gp_set_moment):
        f.argtypes = [P, I, I, I, FP, SZ]
    lib.gp_get_updates.argtypes = [P, ctypes.POINTER(ctypes.c_longlong)]
    lib.gp_set_updates.argtypes = [P, ctypes.c_longlong]
    lib.gp_partition_memory.argtypes = [P] + [ctypes.POINTER(SZ)] * 4
    lib.gp_param_count.argtypes = [P, ctypes.POINTER(SZ)]
    lib.gp_forward_microbatch.argtypes = [P, I, VP, VP, VP, VP]
    lib.gp_forward_microbatch_noalloc.argtypes = [P, I, VP, VP, VP, VP]
    lib.gp_plan_cells.argtypes = [ctypes.POINTER(ctypes.c_double), I, I, ctypes.POINTER(ctypes.c_int),
                                  ctypes.POINTER(ctypes.c_double)]
    lib.gp_backward_microbatch_remat.argtypes = [P, I, VP, VP, VP, VP]
    lib.gp_accumulate_and_step.argtypes = [P, ctypes.c_float, ctypes.POINTER(ctypes.c_double), VP]
    D = ctypes.POINTER(ctypes.c_double)
    lib.gp_timer_select.argtypes = [P, I]
    lib.gp_timer_read.argtypes = [P, I, D, ctypes.POINTER(ctypes.c_long), D, D]
    lib.gp_timer_reset.argtypes = [P]
    lib.gp_timer_sample.argtypes = [P, I]
    lib.gp_mfma_peak.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_double)]
    lib.gp_recomputed_output.argtypes = [P, VP, VP]
    lib.gp_stream_create.argtypes = [ctypes.POINTER(VP)]
    lib.gp_stream_destroy.argtypes = [VP]
    lib.gp_memory_plan.argtypes = [I, I, I, I, ctypes.POINTER(gp_config)] + [ctypes.POINTER(SZ)] * 4
    L, F = ctypes.c_long, ctypes.c_float
    lib.gp_token_logprobs.argtypes = [I, VP, L, I, L, VP, F, F, VP, VP, VP, I, VP, VP, VP, SZ, VP]
    lib.gp_token_logprobs_workspace.argtypes = [I, L, I, I, ctypes.POINTER(SZ)]
    lib.gp_token_logprobs_backward.argtypes = [I, VP, L, I, L, VP, F, F, VP, VP, VP, VP, VP, L, VP]
    lib.gp_grad_norm.argtypes = [I, ctypes.POINTER(gp_grad_tensor), I, F, VP, VP, SZ, VP]
    lib.gp_grad_norm_workspace.argtypes = [I, ctypes.POINTER(SZ)]
    lib.gp_adamw_step.argtypes = [ctypes.POINTER(gp_adamw_tensor), I, ctypes.POINTER(gp_adamw_config),
                                  ctypes.c_longlong, VP, VP, VP]
    lib.gp_backward_microbatch_weighted.argtypes = [P, I, VP, VP, VP, VP, VP, VP]
    lib.gp_get_grad_norm.argtypes = [P, ctypes.POINTER(F)]
    lib.gp_score_sequences.argtypes = [P, VP, VP, VP, F, VP, VP, VP, I, VP, VP, VP]
    lib.gp_distill.argtypes = [I, VP, L, I, L, VP, VP, I, F, F, I, VP, VP, VP, VP, SZ, VP]
    lib.gp_distill_workspace.argtypes = [I, L, I, ctypes.POINTER(SZ)]
    lib.gp_distill_backward.argtypes = [I, VP, L, I, L, VP, VP, I, F, F, I, VP, VP, VP, VP, L, VP]
    C, R = ctypes.POINTER(gp_attention_config), ctypes.POINTER(gp_head_rows)
    lib.gp_attention.argtypes = [C, R, R, R, R, VP, VP, SZ, VP]
    lib.gp_attention_workspace.argtypes = [C, I, ctypes.POINTER(SZ)]
    lib.gp_attention_backward.argtypes = [C, R, R, R, R, VP, R, R, R, R, VP, VP, SZ, VP]
    lib.gp_relative_buckets.argtypes = [I, I, I, ctypes.POINTER(ctypes.c_int)]
    lib.gp_last_error.argtypes = []
    lib.gp_last_error.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name != "gp_last_error":
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def gp_last_error() -> str:
    return load().gp_last_error().decode()


def _check(status):
    if status != GP_OK:
        raise GpError(status, gp_last_error())


def _fptr(a):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))


# --- one function per C entry point, same names -------------------------------
def gp_partition_create(layers, d_model, d_ff, heads):
    h = ctypes.c_void_p()
    _check(load().gp_partition_create(layers, d_model, d_ff, heads, ctypes.byref(h)))
    return h


def gp_partition_configure(h, cfg: gp_config):
    _check(load().gp_partition_configure(h, ctypes.byref(cfg)))


def gp_partition_destroy(h):
    _check(load().gp_partition_destroy(h))


def gp_set_param(h, layer, pid, host):
    """host: C-contiguous float32 numpy array."""
    _check(load().gp_set_param(h, layer, pid, _fptr(host), host.size))


def gp_get_param(h, layer, pid, host):
    _check(load().gp_get_param(h, layer, pid, _fptr(host), host.size))


def gp_get_grad(h, layer, pid, host):
    _check(load().gp_get_grad(h, layer, pid, _fptr(host), host.size))


def gp_get_moment(h, layer, pid, which, host):
    _check(load().gp_get_moment(h, layer, pid, which, _fptr(host), host.size))


def gp_set_moment(h, layer, pid, which, host):
    """host: C-contiguous float32 numpy array."""
    _check(load().gp_set_moment(h, layer, pid, which, _fptr(host), host.size))


def gp_get_updates(h):
    v = ctypes.c_longlong()
    _check(load().gp_get_updates(h, ctypes.byref(v)))
    return v.value


def gp_set_updates(h, updates):
    _check(load().gp_set_updates(h, updates))


def gp_partition_memory(h):
    v = [ctypes.c_size_t() for _ in range(4)]
    _check(load().gp_partition_memory(h, *[ctypes.byref(x) for x in v]))
    return dict(params=v[0].value, grads=v[1].value, stash=v[2].value, workspace=v[3].value)


def gp_memory_plan(layers, d_model, d_ff, heads, cfg: gp_config):
    """Byte counts of a partition configured with cfg, computed on the host."""
    v = [ctypes.c_size_t() for _ in range(4)]
    _check(load().gp_memory_plan(layers, d_model, d_ff, heads, ctypes.byref(cfg), *[ctypes.byref(x) for x in v]))
    return dict(params=v[0].value, grads=v[1].value, stash=v[2].value, workspace=v[3].value)


def gp_plan_cells(costs, cells):
    """Least-variance split of the layers (costs: 1-D float array) into
    `cells` cells; returns (first layer of each cell, variance)."""
    import numpy as np
    c = np.ascontiguousarray(costs, dtype=np.float64)
    first = (ctypes.c_int * max(cells, 1))()
    var = ctypes.c_double()
    _check(load().gp_plan_cells(c.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), c.size, cells, first,
                                ctypes.byref(var)))
    return [int(v) for v in first[:cells]], var.value


def gp_param_count(h):
    v = ctypes.c_size_t()
    _check(load().gp_param_count(h, ctypes.byref(v)))
    return v.value


def gp_forward_microbatch(h, mb, x, mem, y, stream):
    _check(load().gp_forward_microbatch(h, mb, x, mem, y, stream))


def gp_forward_microbatch_noalloc(h, mb, x, mem, y, stream):
    _check(load().gp_forward_microbatch_noalloc(h, mb, x, mem, y, stream))


def gp_backward_microbatch_remat(h, mb, dy_or_target, dx, dmem, stream):
    _check(load().gp_backward_microbatch_remat(h, mb, dy_or_target, dx, dmem, stream))


def gp_backward_microbatch_weighted(h, mb, tokens, dlogp, dentropy, dx, dmem, stream):
    _check(load().gp_backward_microbatch_weighted(h, mb, tokens, dlogp, dentropy, dx, dmem, stream))


def gp_accumulate_and_step(h, lr, want_loss, stream):
    if want_loss:
        v = ctypes.c_double()
        _check(load().gp_accumulate_and_step(h, lr, ctypes.byref(v), stream))
        return v.value
    _check(load().gp_accumulate_and_step(h, lr, None, stream))
    return None


def gp_get_grad_norm(h):
    v = ctypes.c_float()
    _check(load().gp_get_grad_norm(h, ctypes.byref(v)))
    return v.value


def gp_score_sequences(h, x, mem, tokens, scale, logp, lse, entropy, top, top_ids, top_logp, stream):
    _check(load().gp_score_sequences(h, x, mem, tokens, scale, logp, lse, entropy, top, top_ids, top_logp, stream))


def gp_timer_select(h, role):
    _check(load().gp_timer_select(h, role))


def gp_timer_read(h, role):
    """(milliseconds, launches, FLOPs, bytes) of one launch role."""
    ms, fl, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
    n = ctypes.c_long()
    _check(load().gp_timer_read(h, role, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl), ctypes.byref(by)))
    return ms.value, n.value, fl.value, by.value


def gp_timer_reset(h):
    _check(load().gp_timer_reset(h))


def gp_timer_sample(h, every):
    _check(load().gp_timer_sample(h, every))


def gp_stream_create():
    """A non-blocking stream of default priority (its raw handle)."""
    s = ctypes.c_void_p()
    _check(load().gp_stream_create(ctypes.byref(s)))
    return s.value


def gp_stream_destroy(stream):
    _check(load().gp_stream_destroy(stream))


def gp_recomputed_output(h, y, stream):
    """y: device address of an [n, S, D] buffer in the partition dtype."""
    _check(load().gp_recomputed_output(h, y, stream))


def gp_token_logprobs(dtype, logits, rows, vocab, ld, tokens, scale, clip, logp, lse, entropy, top, top_ids, top_logp,
                      ws, ws_bytes, stream):
    _check(load().gp_token_logprobs(dtype, logits, rows, vocab, ld, tokens, scale, clip, logp, lse, entropy, top,
                                    top_ids, top_logp, ws, ws_bytes, stream))


def gp_token_logprobs_workspace(dtype, rows, vocab, top):
    """Bytes of scratch with which gp_token_logprobs is fastest."""
    v = ctypes.c_size_t()
    _check(load().gp_token_logprobs_workspace(dtype, rows, vocab, top, ctypes.byref(v)))
    return v.value


def gp_token_logprobs_backward(dtype, logits, rows, vocab, ld, tokens, scale, clip, lse, entropy, dlogp, dentropy,
                               dlogits, ldd, stream):
    _check(load().gp_token_logprobs_backward(dtype, logits, rows, vocab, ld, tokens, scale, clip, lse, entropy, dlogp,
                                             dentropy, dlogits, ldd, stream))


def gp_distill(dtype, logits, rows, vocab, ld, ids, teacher, top, scale, clip, rest, loss, lse, rest_lse, ws, ws_bytes,
               stream):
    _check(load().gp_distill(dtype, logits, rows, vocab, ld, ids, teacher, top, scale, clip, rest, loss, lse, rest_lse, ws,
                             ws_bytes, stream))


def gp_distill_workspace(dtype, rows, vocab):
    """Bytes of scratch with which gp_distill is fastest."""
    v = ctypes.c_size_t()
    _check(load().gp_distill_workspace(dtype, rows, vocab, ctypes.byref(v)))
    return v.value


def gp_distill_backward(dtype, logits, rows, vocab, ld, ids, teacher, top, scale, clip, rest, lse, rest_lse, dloss, dlogits,
                        ldd, stream):
    _check(load().gp_distill_backward(dtype, logits, rows, vocab, ld, ids, teacher, top, scale, clip, rest, lse, rest_lse,
                                      dloss, dlogits, ldd, stream))


def gp_grad_norm(dtype, grads, n, max_norm, norm_factor, ws, ws_bytes, stream):
    """grads: an array of gp_grad_tensor."""
    _check(load().gp_grad_norm(dtype, grads, n, max_norm, norm_factor, ws, ws_bytes, stream))


def gp_grad_norm_workspace(n):
    v = ctypes.c_size_t()
    _check(load().gp_grad_norm_workspace(n, ctypes.byref(v)))
    return v.value


def gp_adamw_step(tensors, n, cfg: gp_adamw_config, step, step_dev, factor, stream):
    """tensors: an array of gp_adamw_tensor."""
    _check(load().gp_adamw_step(tensors, n, ctypes.byref(cfg), step, step_dev, factor, stream))


def gp_attention(cfg: gp_attention_config, q, k, v, out, lse, ws, ws_bytes, stream):
    """q, k, v, out: gp_head_rows."""
    _check(load().gp_attention(cfg, q, k, v, out, lse, ws, ws_bytes, stream))


def gp_attention_workspace(cfg: gp_attention_config, backward):
    v = ctypes.c_size_t()
    _check(load().gp_attention_workspace(cfg, backward, ctypes.byref(v)))
    return v.value


def gp_attention_backward(cfg: gp_attention_config, q, k, v, out, lse, dout, dq, dk, dv, dbias, ws, ws_bytes, stream):
    """q, k, v, out (or None), dout, dq, dk, dv: gp_head_rows."""
    _check(load().gp_attention_backward(cfg, q, k, v, out, lse, dout, dq, dk, dv, dbias, ws, ws_bytes, stream))


def gp_relative_buckets(buckets, max_distance, bidirectional):
    """Bucket of each distance from -max_distance to max_distance (a list)."""
    v = (ctypes.c_int * (2 * max(0, min(max_distance, GP_DISTANCE_MAX)) + 1))()
    _check(load().gp_relative_buckets(buckets, max_distance, bidirectional, v))
    return list(v)


def gp_mfma_peak(stream=None):
    """Sustained bf16 MFMA-loop rate of the current device, TFLOP/s."""
    t = ctypes.c_double()
    _check(load().gp_mfma_peak(stream, ctypes.byref(t)))
    return t.value
