"""Torch-facing operators on the caller's own tensors (marshalling only).

Beside the partition's own head and update: log probabilities of given tokens
with entropy and alternatives (``token_logprobs``) and their gradient
(``token_logprobs_backward``), the divergence from a teacher's most likely tokens
(``distill``) and its gradient (``distill_backward``), the norm over many gradients (``grad_norm``),
AdamW over many tensors with states in 32 or 8 bits (``AdamW``), attention to keys of
another length with a learned relative position bias (``attention``, ``RelativeBias``)
and its gradients (``attention_backward``).  Every step of
the work runs in libgp.so, on the current stream of the tensors' device;
results and scratch memory come from torch's allocator.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional, Sequence, Union

import numpy as np
import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

from . import gp

DTYPE = {torch.float32: gp.GP_F32, torch.bfloat16: gp.GP_BF16}


class TokenLogprobs(NamedTuple):
    logp: Optional[torch.Tensor]      # fp32 [rows]; None without tokens
    lse: torch.Tensor                 # fp32 [rows]
    entropy: torch.Tensor             # fp32 [rows]
    top_ids: Optional[torch.Tensor]   # int32 [rows, top]; None for top = 0
    top_logp: Optional[torch.Tensor]  # fp32 [rows, top]


def _on(device, call):
    """call(stream) with the device current and its current stream's handle."""
    i = device.index
    if i == torch._C._cuda_getDevice():
        call(torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            call(torch._C._cuda_getCurrentRawStream(i))


def _gpu(t):
    if not t.is_cuda:
        raise ValueError("tensors must be on a GPU")
    return t.device


def _ptr(t):
    return None if t is None else t.data_ptr()


def _rows(name, t):
    """(rows, vocab, ld) of a matrix whose rows are contiguous."""
    if t.dim() != 2 or t.dtype not in DTYPE:
        raise ValueError(f"{name} must be a matrix in float32 or bfloat16")
    rows, vocab = t.shape
    if vocab > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    ld = t.stride(0) if rows > 1 else max(vocab, t.stride(0))
    if ld < vocab:
        raise ValueError(f"{name}: rows must not overlap")
    return rows, vocab, ld


def _no_graph(*tensors, gradient="token_logprobs_backward"):
    """The operators build no autograd graph: an input whose gradient, or whose tangent in forward mode, would be lost is refused."""
    if forward_ad._current_level >= 0:  # within a dual_level
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError("forward-mode differentiation is not supported here: an input has a tangent")
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("no autograd graph is built here: detach the inputs, or call under torch.no_grad(), and "
                                 f"take the gradient from {gradient}")


def _vector(name, t, rows, dtype, device):
    if t is not None and (t.dtype != dtype or t.dim() != 1 or t.numel() != rows or t.device != device
                          or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} vector of one value per row on {device}")


def token_logprobs(logits, tokens=None, scale=1.0, clip=0.0, top=0) -> TokenLogprobs:
    """gp_token_logprobs of rows of logits [rows, vocab] (a row stride is fine)
    and int32 tokens [rows] (gp.GP_NO_TOKEN where there is none; None: no
    logp).  scale: 1 / temperature; clip: the head's logit clip, 0 = off (it lifts a
    masked logit to -clip: clip before masking instead).  Not
    differentiable by itself: logits that require a gradient are refused unless
    autograd is off."""
    _no_graph(logits)
    rows, vocab, ld = _rows("logits", logits)
    dev, dt = _gpu(logits), DTYPE[logits.dtype]
    _vector("tokens", tokens, rows, torch.int32, dev)
    need = gp.gp_token_logprobs_workspace(dt, rows, vocab, top)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    logp, lse, entropy = torch.empty((3, rows), dtype=torch.float32, device=dev).unbind(0)
    if tokens is None:
        logp = None
    top_ids = torch.empty((rows, top), dtype=torch.int32, device=dev) if top else None
    top_logp = torch.empty((rows, top), dtype=torch.float32, device=dev) if top else None
    _on(dev, lambda stream: gp.gp_token_logprobs(
        dt, logits.data_ptr(), rows, vocab, ld, _ptr(tokens), scale, clip, _ptr(logp), lse.data_ptr(),
        entropy.data_ptr(), top, _ptr(top_ids), _ptr(top_logp), _ptr(ws), need, stream))
    return TokenLogprobs(logp, lse, entropy, top_ids, top_logp)


def _gradient_of(logits, vocab, ld, out):
    """(where the logits' gradient goes, its row stride)."""
    if out is None:
        return torch.empty(logits.shape, dtype=logits.dtype, device=logits.device), vocab
    if out is logits:
        return out, ld
    if out.dtype != logits.dtype or out.shape != logits.shape or out.device != logits.device:
        raise ValueError("out must have the type, shape and device of the logits")
    return out, _rows("out", out)[2]


def token_logprobs_backward(logits, tokens, lse, entropy=None, dlogp=None, dentropy=None, scale=1.0, clip=0.0,
                            out=None):
    """gp_token_logprobs_backward: the gradient of sum dlogp logp + dentropy
    entropy with respect to the logits.  out: where it goes (may be logits
    itself); allocated otherwise."""
    _no_graph(logits, lse, entropy, dlogp, dentropy, out)
    rows, vocab, ld = _rows("logits", logits)
    dev = _gpu(logits)
    _vector("tokens", tokens, rows, torch.int32, dev)
    for name, t in (("lse", lse), ("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy)):
        _vector(name, t, rows, torch.float32, dev)
    out, ldd = _gradient_of(logits, vocab, ld, out)
    _on(dev, lambda stream: gp.gp_token_logprobs_backward(
        DTYPE[logits.dtype], logits.data_ptr(), rows, vocab, ld, _ptr(tokens), scale, clip, _ptr(lse), _ptr(entropy),
        _ptr(dlogp), _ptr(dentropy), out.data_ptr(), ldd, stream))
    increment_version(out)  # a graph that saved it must not be walked back with what it holds now
    return out


class Distillation(NamedTuple):
    loss: torch.Tensor                # fp32 [rows]
    lse: torch.Tensor                 # fp32 [rows]
    rest_lse: Optional[torch.Tensor]  # fp32 [rows]; None without rest


def _teacher(ids, teacher, rows, device):
    """Tokens named per row."""
    for name, t, kind in (("ids", ids, torch.int32), ("teacher", teacher, torch.float32)):
        if t.dim() != 2 or t.shape[0] != rows or t.shape != ids.shape or t.dtype != kind or t.device != device or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {kind} [rows, top] on {device}")
    return ids.shape[1]


def distill(logits, ids, teacher, scale=1.0, clip=0.0, rest=True) -> Distillation:
    """gp_distill: the divergence of rows of logits [rows, vocab] (a row stride is
    fine) from a teacher's log probabilities, fp32 [rows, top], of the tokens ids, int32 [rows, top]
    (``token_logprobs(teacher_logits, top=n)`` gives both; gp.GP_NO_TOKEN where a row names
    fewer).  rest: what the teacher gives to the other tokens is one more outcome; without
    it the named tokens' probabilities are normalised.  scale, clip: as token_logprobs.  Not
    differentiable by itself: distill_backward gives the gradient."""
    _no_graph(logits, teacher, gradient="distill_backward")
    rows, vocab, ld = _rows("logits", logits)
    dev, dt = _gpu(logits), DTYPE[logits.dtype]
    top = _teacher(ids, teacher, rows, dev)
    need = gp.gp_distill_workspace(dt, rows, vocab)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    loss, lse, rest_lse = torch.empty((3, rows), dtype=torch.float32, device=dev).unbind(0)
    if not rest:
        rest_lse = None
    _on(dev, lambda stream: gp.gp_distill(
        dt, logits.data_ptr(), rows, vocab, ld, ids.data_ptr(), teacher.data_ptr(), top, scale, clip, rest, loss.data_ptr(),
        lse.data_ptr(), _ptr(rest_lse), _ptr(ws), need, stream))
    return Distillation(loss, lse, rest_lse)


def distill_backward(logits, ids, teacher, lse, dloss, rest_lse=None, scale=1.0, clip=0.0, rest=True, out=None):
    """gp_distill_backward: the gradient of sum dloss loss with respect to the
    logits, from the lse and rest_lse that ``distill`` gave for the same arguments.  out: where it
    goes (may be logits itself); allocated otherwise."""
    _no_graph(logits, teacher, lse, dloss, rest_lse, out, gradient="this call's result")
    rows, vocab, ld = _rows("logits", logits)
    dev = _gpu(logits)
    top = _teacher(ids, teacher, rows, dev)
    for name, t in (("lse", lse), ("dloss", dloss), ("rest_lse", rest_lse)):
        _vector(name, t, rows, torch.float32, dev)
    out, ldd = _gradient_of(logits, vocab, ld, out)
    _on(dev, lambda stream: gp.gp_distill_backward(
        DTYPE[logits.dtype], logits.data_ptr(), rows, vocab, ld, ids.data_ptr(), teacher.data_ptr(), top, scale, clip, rest,
        _ptr(lse), _ptr(rest_lse), _ptr(dloss), out.data_ptr(), ldd, stream))
    increment_version(out)
    return out


def _fits(t, like):
    """Of the same shape, up to dimensions of 1, or one of them flat: a transposed tensor has as many elements too."""
    if t.shape == like.shape:
        return True
    a, b = ([n for n in x.shape if n != 1] for x in (t, like))
    return t.numel() == like.numel() and (a == b or len(a) == 1 or len(b) == 1 or t.numel() == 0)


def _same(name, tensors, like=None):
    """Tensors of one type on one GPU, each contiguous (and of the shapes of `like`)."""
    tensors = list(tensors)
    if tensors:
        kind, dev = tensors[0].dtype, tensors[0].get_device()
        if dev < 0 or any(t.dtype != kind or t.get_device() != dev or not t.is_contiguous() for t in tensors):
            raise ValueError(f"{name} must be contiguous tensors of one type on one GPU")
    if like is not None and (len(tensors) != len(like) or not all(map(_fits, tensors, like))):
        raise ValueError(f"{name} must match the parameters one by one")
    return tensors


def _records(struct, n, **columns):
    """An array of n ctypes structures from columns of whole numbers or floats, and what keeps it alive."""
    rows = np.zeros(n, dtype=np.dtype(struct))
    for name, values in columns.items():
        rows[name] = values
    return rows, ctypes.cast(rows.ctypes.data, ctypes.POINTER(struct))


def _addresses(tensors):
    return list(map(torch.Tensor.data_ptr, tensors))


def _spans(rows, **bytes_each):
    """Starts and ends, by start, of what each column's addresses and the bytes of each tensor make; empty ones left out."""
    start = np.concatenate([rows[k] for k in bytes_each]).astype(np.int64)
    size = np.concatenate([np.broadcast_to(b, rows.shape) for b in bytes_each.values()])
    order = np.argsort(np.where(size > 0, start, -1), kind="stable")[np.count_nonzero(size == 0):]
    return start[order], (start + size)[order]


class TensorList:
    """Gradients that a program passes again and again: checked and listed once,
    and again where one has been given other storage (``.data``, ``set_``).  Holds
    the tensors."""

    def __init__(self, tensors: Sequence[torch.Tensor]):
        self.tensors = list(tensors)
        self._list(_addresses(self.tensors))

    def _list(self, addresses):
        _same("gradients", self.tensors)
        if not self.tensors or self.tensors[0].dtype not in DTYPE:
            raise ValueError("a TensorList needs float32 or bfloat16 tensors")
        self.dtype = DTYPE[self.tensors[0].dtype]
        self.scratch = gp.gp_grad_norm_workspace(len(self.tensors))  # bytes that grad_norm takes
        self._rows, self.array = _records(gp.gp_grad_tensor, len(self.tensors), grad=addresses,
                                          count=[t.numel() for t in self.tensors])
        self._at = addresses

    def follow(self):
        """Lists the tensors anew if one has moved."""
        now = _addresses(self.tensors)
        if now != self._at:
            self._list(now)
        return self


def grad_norm(grads: Union[TensorList, Sequence[torch.Tensor]], max_norm=float("inf")):
    """fp32 [2] on the device: the 2-norm over all the tensors, and the factor
    min(1, max_norm / norm) that clips them (NaN where the norm is not finite)."""
    g = grads.follow() if isinstance(grads, TensorList) else TensorList(grads)
    dev, need = g.tensors[0].device, g.scratch
    out = torch.empty(2, dtype=torch.float32, device=dev)
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _on(dev, lambda stream: gp.gp_grad_norm(g.dtype, g.array, len(g.tensors), max_norm, out.data_ptr(), ws.data_ptr(),
                                            need, stream))
    return out


class AdamW:
    """AdamW over a list of parameters, one gp_adamw_step per ``step``.

    params: contiguous fp32 or bf16 tensors.  grads: one per parameter, read at
    every step (``bind_grads`` names others); they, the states and the copies have
    their parameter's shape or are flat.  state_bits: 32, or 8 (e4m3 values
    with an fp32 scale per 256 elements, v held as its square root); the states
    start at zero, or m, v (and m_scale, v_scale) are taken as they are, of the
    types that ``m`` and ``v`` of another AdamW have.  copies: bf16 tensors that
    receive the updated fp32 parameters.  weight_decay: a number or one per
    parameter.  steps: updates done before.  capturable: the step counter lives
    on the device (``step_dev``), as a step recorded into a graph needs.

    Parameters, gradients and copies that are given other storage (``.data``,
    ``set_``, a module's ``to``) are followed at the next step, and refused if they
    no longer match.  The states stay in the storage that they had here: change them in
    place (``copy_``)."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m=None, v=None, m_scale=None,
                 v_scale=None, copies=None, state_bits: Optional[int] = None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8,
                 weight_decay: Union[float, Sequence[float]] = 0.0, seed=0, steps=0, capturable=False):
        self.params = _same("params", params)
        if not self.params or self.params[0].dtype not in DTYPE:
            raise ValueError("params must be float32 or bfloat16 tensors")
        if state_bits is None:
            state_bits = 8 if m and m[0].dtype == torch.float8_e4m3fn else 32
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 32 or 8")
        if steps < 0:
            raise ValueError("steps must not be negative")
        dev, n = self.params[0].device, len(self.params)
        kind = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        if (m is None) != (v is None):
            raise ValueError("m and v come together")
        if m is None:
            m = [torch.zeros(p.shape, dtype=kind, device=dev) for p in self.params]
            v = [torch.zeros(p.shape, dtype=kind, device=dev) for p in self.params]
        self.m, self.v = _same("m", m, self.params), _same("v", v, self.params)
        if any(t.dtype != kind or t.device != dev for t in self.m + self.v):
            raise ValueError(f"m and v must be {kind} on {dev}")
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            blocks = [(p.numel() + gp.GP_STATE_BLOCK - 1) // gp.GP_STATE_BLOCK for p in self.params]
            if m_scale is None and v_scale is None:
                m_scale, v_scale = ([torch.zeros(b, device=dev) for b in blocks] for _ in range(2))
            if m_scale is None or v_scale is None:
                raise ValueError("m_scale and v_scale come together")
            self.m_scale, self.v_scale = _same("m_scale", m_scale), _same("v_scale", v_scale)
            for s in (self.m_scale, self.v_scale):
                if [t.numel() for t in s] != blocks or any(t.dtype != torch.float32 or t.device != dev for t in s):
                    raise ValueError("m_scale and v_scale must hold one float32 per 256 elements of their parameter")
        elif m_scale is not None or v_scale is not None:
            raise ValueError("scales belong to 8-bit states")
        self.copies = None if copies is None else list(copies)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        if len(decay) != n:
            raise ValueError("weight_decay must be a number or one per parameter")
        columns = dict(count=[p.numel() for p in self.params], weight_decay=decay, m=_addresses(self.m),
                       v=_addresses(self.v))
        if state_bits == 8:
            columns.update(m_scale=_addresses(self.m_scale), v_scale=_addresses(self.v_scale))
        self._rows, self.array = _records(gp.gp_adamw_tensor, n, **columns)
        # the states' storage lives as long as their addresses here
        self._states = [t.detach() for t in [*self.m, *self.v, *(self.m_scale or ()), *(self.v_scale or ())]]
        self.cfg = gp.gp_adamw_config(DTYPE[self.params[0].dtype], 0, state_bits, seed, lr, betas[0], betas[1], eps)
        self.device, self.steps = dev, steps
        self.step_dev = torch.full((1,), steps, dtype=torch.int64, device=dev) if capturable else None
        self._list(grads)

    def _list(self, grads):
        """The addresses of parameters, copies and gradients as they are now, checked against the states'."""
        self._written_at = None  # whatever is refused below is looked at again
        dev, states = self.device, self._states[:len(self.params)]
        params = _same("params", self.params, states)
        copies = [] if self.copies is None else _same("copies", self.copies, states)
        if params[0].dtype not in DTYPE or params[0].device != dev:
            raise ValueError(f"params must be float32 or bfloat16 on {dev}")
        if copies and (copies[0].dtype != torch.bfloat16 or copies[0].device != dev):
            raise ValueError(f"copies must be bfloat16 on {dev}")
        at, copies_at = _addresses(params), _addresses(copies)
        self.cfg.param_dtype = DTYPE[params[0].dtype]
        self._rows["param"] = at
        if copies:
            self._rows["copy"] = copies_at
        n = self._rows["count"]
        state = n * states[0].element_size()
        columns = dict(param=n * params[0].element_size(), m=state, v=state)
        if self.m_scale is not None:
            columns["m_scale"] = columns["v_scale"] = -(-n // gp.GP_STATE_BLOCK) * 4
        if copies:
            columns["copy"] = n * 2
        self._starts, self._ends = _spans(self._rows, **columns)
        if (self._starts[1:] < self._ends[:-1]).any():
            raise ValueError("parameters, states, scales and copies must not share memory")
        self._list_grads(grads)
        self._written, self._written_at = params + copies, at + copies_at

    def bind_grads(self, grads: Sequence[torch.Tensor]):
        """The gradients that the next steps read."""
        if _addresses(self._written) != self._written_at:
            self._list(grads)
        else:
            self._list_grads(grads)

    def _list_grads(self, grads):
        grads = _same("grads", grads, self.params)
        if grads[0].dtype not in DTYPE or grads[0].device != self.device:
            raise ValueError("grads must be float32 or bfloat16 on the parameters' device")
        at = _addresses(grads)
        n = self._rows["count"] * grads[0].element_size()
        start = np.array(at, dtype=np.int64)
        # the first output that ends behind a gradient's start begins behind its end
        behind = np.searchsorted(self._ends, start, side="right")
        if ((start + n > np.append(self._starts, np.iinfo(np.int64).max)[behind]) & (n > 0)).any():
            raise ValueError("gradients must not share memory with what a step writes")
        self.grads = grads
        self.cfg.grad_dtype = DTYPE[grads[0].dtype]
        self._grads_at = at
        self._rows["grad"] = at

    def step(self, lr: Optional[float] = None, factor: Optional[torch.Tensor] = None):
        """One update.  factor: fp32 on the device, multiplied into every
        gradient (``grad_norm(...)[1:]``); a NaN leaves everything as it was.
        The host's count ``steps`` goes up either way, for the factor stays on the
        device: the bias corrections that follow count a skipped update, unless
        capturable, where the device's counter does not.  A captured step keeps
        the lr, seed and addresses it was captured with."""
        if lr is not None:
            self.cfg.lr = lr
        dev = self.device
        if factor is not None and (factor.dtype != torch.float32 or factor.numel() != 1 or factor.device != dev):
            raise ValueError("factor must be one float32 on the parameters' device")
        if _addresses(self._written) != self._written_at or _addresses(self.grads) != self._grads_at:
            self._list(self.grads)
        host = 0 if self.step_dev is not None else self.steps + 1
        _on(dev, lambda stream: gp.gp_adamw_step(self.array, len(self.params), self.cfg, host, _ptr(self.step_dev),
                                                 _ptr(factor), stream))
        increment_version(self._written)  # parameters that a graph saved are not those it would walk back with
        self.steps += 1


class RelativeBias:
    """A learned bias by relative position: table[h, bucket(key - query)] is
    added to the scores of head h.  table: contiguous fp32 [heads, buckets], read at every
    call (an optimiser updates it in place).  The buckets are gp_relative_buckets': half of
    one side's hold one distance each, the others grow with the logarithm up to max_distance,
    beyond which all share the last; bidirectional: one half for keys behind the query.  The map of
    distances is made here, once: another number of buckets or distance takes another
    RelativeBias (table may be replaced by one of the same shape)."""

    def __init__(self, table: torch.Tensor, max_distance=128, bidirectional=True):
        if table.dim() != 2 or table.dtype != torch.float32:
            raise ValueError("table must be float32 [heads, buckets]")
        dev = _gpu(table)
        self.table = table
        self._buckets, self._max_distance, self._bidirectional = table.shape[1], max_distance, bidirectional
        of = gp.gp_relative_buckets(table.shape[1], max_distance, bidirectional)
        self._bucket_of = torch.tensor(of, dtype=torch.int32).to(dev)

    # the kernels read 2 max_distance + 1 places of bucket_of
    max_distance = property(lambda self: self._max_distance)
    bidirectional = property(lambda self: self._bidirectional)
    bucket_of = property(lambda self: self._bucket_of)


class Attention(NamedTuple):
    out: torch.Tensor  # [batch, q_len, heads, head_dim], of the type of q
    lse: torch.Tensor  # fp32 [batch, heads, q_len]


class AttentionGrads(NamedTuple):
    dq: torch.Tensor
    dk: torch.Tensor
    dv: torch.Tensor
    dbias: Optional[torch.Tensor]  # fp32 [heads, buckets]; None without a bias


def _head_rows(name, t, kind, device, shape):
    """gp_head_rows of a tensor [batch, len, heads, head_dim] of this type, on the device of this index."""
    if t.shape != shape or t.dtype != kind or t.get_device() != device:
        raise ValueError(f"{name} must be {list(shape)} in {kind} on GPU {device}")
    a, b, c, d = t.stride()
    if d != 1 and shape[3] > 1:
        raise ValueError(f"{name}: the features of a head must be adjacent")
    return gp.gp_head_rows(t.data_ptr(), a, b, c)


@functools.lru_cache(maxsize=256)
def _attention_bytes(backward, *sizes):
    """Bytes of scratch: they depend on the sizes alone."""
    cfg = gp.gp_attention_config(*sizes[:7], 0, 1.0)
    if sizes[7]:
        cfg.bias = cfg.bucket_of = 16
        cfg.buckets, cfg.max_distance = sizes[7:]
    return gp.gp_attention_workspace(cfg, backward)


def _attention(q, k, v, q_lens, k_lens, q_starts, causal, scale, bias, backward):
    """(config, gp_head_rows of q, k and v, bytes of scratch)."""
    kind = q.dtype
    if q.dim() != 4 or k.dim() != 4 or kind not in DTYPE:
        raise ValueError("q, k and v must be [batch, len, heads, head_dim] in float32 or bfloat16")
    shape, like = q.shape, k.shape
    B, Sq, H, dh = shape
    _, Sk, K, _ = like
    if like[0] != B or like[3] != dh:
        raise ValueError("q, k and v must have the same batch and head_dim")
    dev = _gpu(q)
    at = dev.index
    rows = (_head_rows("q", q, kind, at, shape), _head_rows("k", k, kind, at, like), _head_rows("v", v, kind, at, like))
    if q_lens is not None:
        _vector("q_lens", q_lens, B, torch.int32, dev)
    if k_lens is not None:
        _vector("k_lens", k_lens, B, torch.int32, dev)
    if q_starts is not None:
        _vector("q_starts", q_starts, B, torch.int32, dev)
    dt = DTYPE[kind]
    cfg = gp.gp_attention_config(dt, B, H, K, Sq, Sk, dh, causal, dh ** -0.5 if scale is None else scale, _ptr(q_lens),
                                 _ptr(k_lens), _ptr(q_starts))
    buckets = distance = 0
    if bias is not None:
        table, of, buckets, distance = bias.table, bias._bucket_of, bias._buckets, bias._max_distance
        if table.dtype != torch.float32 or table.shape != (H, buckets) or table.get_device() != at or not table.is_contiguous():
            raise ValueError(f"the bias must have a contiguous float32 table of {H} heads and {buckets} buckets on {dev}")
        if of.get_device() != at:
            raise ValueError(f"the bias was made on {of.device}")
        if of.numel() != 2 * distance + 1 or not of.is_contiguous():
            raise ValueError("bucket_of has been changed in length")
        cfg.bias, cfg.bucket_of, cfg.buckets, cfg.max_distance = table.data_ptr(), of.data_ptr(), buckets, distance
    return cfg, rows, _attention_bytes(backward, dt, B, H, K, Sq, Sk, dh, buckets, distance)


def attention(q, k, v, q_lens=None, k_lens=None, q_starts=None, causal=False, scale=None,
              bias: Optional[RelativeBias] = None) -> Attention:
    """gp_attention: softmax(scale q k^T + bias) v of queries [batch, q_len,
    heads, head_dim] over keys and values [batch, k_len, kv_heads, head_dim] of any strides
    (features adjacent), kv_heads dividing heads.  q_lens, k_lens: int32 [batch], rows in
    use of each sequence; q_starts: int32 [batch], position of the first query among the keys
    (0), for causal and the bias.  scale: 1 / sqrt(head_dim) unless given.  Not differentiable
    by itself: attention_backward gives the gradients."""
    _no_graph(q, k, v, None if bias is None else bias.table, gradient="attention_backward")
    cfg, rows, need = _attention(q, k, v, q_lens, k_lens, q_starts, causal, scale, bias, 0)
    dev, (B, Sq, H, dh) = q.device, q.shape
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    lse = torch.empty_strided((B, H, Sq), (H * Sq, Sq, 1), dtype=torch.float32, device=dev)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    o = gp.gp_head_rows(out.data_ptr(), Sq * H * dh, H * dh, dh)
    _on(dev, lambda stream: gp.gp_attention(cfg, *rows, o, lse.data_ptr(), _ptr(ws), need, stream))
    return Attention(out, lse)


def attention_backward(q, k, v, out, lse, dout, q_lens=None, k_lens=None, q_starts=None, causal=False, scale=None,
                       bias: Optional[RelativeBias] = None, grads=None) -> AttentionGrads:
    """gp_attention_backward: the gradients of sum dout out with respect to q, k,
    v and the bias's table, from the out and lse that ``attention`` gave for the same
    arguments.  out=None: where it was not kept; slower.  grads: (dq, dk, dv), tensors of
    the shapes of q, k and v that receive them; allocated otherwise."""
    _no_graph(q, k, v, out, lse, dout, None if bias is None else bias.table, *(grads or ()), gradient="this call's results")
    cfg, rows, need = _attention(q, k, v, q_lens, k_lens, q_starts, causal, scale, bias, 1)
    dev, kind, shape, like = q.device, q.dtype, q.shape, k.shape
    at = dev.index
    if lse.shape != (shape[0], shape[2], shape[1]) or lse.dtype != torch.float32 or lse.get_device() != at or not lse.is_contiguous():
        raise ValueError("lse must be contiguous float32 [batch, heads, q_len], as attention gives it")
    o = None if out is None else _head_rows("out", out, kind, at, shape)
    g = _head_rows("dout", dout, kind, at, shape)
    if grads is None:
        grads = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v)]
    dq, dk, dv = grads
    to = (_head_rows("dq", dq, kind, at, shape), _head_rows("dk", dk, kind, at, like), _head_rows("dv", dv, kind, at, like))
    dbias = None if bias is None else torch.empty_like(bias.table)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _on(dev, lambda stream: gp.gp_attention_backward(cfg, *rows, o, lse.data_ptr(), g, *to, _ptr(dbias), _ptr(ws), need,
                                                     stream))
    increment_version([dq, dk, dv])
    return AttentionGrads(dq, dk, dv, dbias)
