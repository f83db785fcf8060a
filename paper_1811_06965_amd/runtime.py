"""Torch-facing driver of one partition (marshalling only).

Torch provides device memory and the stream; every step of the partition's
work runs in libgp.so.  ``Partition.step`` issues GPipe's schedule for one
mini-batch (Section 2.2): M forwards in order, M re-materialising backwards in
reverse order, then the one synchronous update.
"""
from __future__ import annotations

from typing import Dict, List, Optional

import numpy as np
import torch

from . import gp
from .ops import TokenLogprobs

# One second stream per device for the odd micro-batches, created by the
# library once per process (a stream from torch's pool may share a hardware
# queue with one of the library's streams).
_SECOND_STREAM: Dict[int, "torch.cuda.ExternalStream"] = {}


def second_stream():
    dev = torch.cuda.current_device()
    if dev not in _SECOND_STREAM:
        _SECOND_STREAM[dev] = torch.cuda.ExternalStream(gp.gp_stream_create(), device=dev)
    return _SECOND_STREAM[dev]


DTYPES = {"f32": (gp.GP_F32, torch.float32), "bf16": (gp.GP_BF16, torch.bfloat16)}
KINDS = {"encoder": gp.GP_ENCODER, "decoder": gp.GP_DECODER_CROSS}
LOSSES = {"none": gp.GP_LOSS_NONE, "mse": gp.GP_LOSS_MSE, "xent_ls": gp.GP_LOSS_XENT_LS}
OPTIMIZERS = {"sgd": gp.GP_OPT_SGD, "rmsprop": gp.GP_OPT_RMSPROP, "adamw": gp.GP_OPT_ADAMW}


def make_config(cfg, micro: Optional[int] = None, check_finite: bool = False,
                keep_activations: bool = False) -> gp.gp_config:
    M = cfg.micro if micro is None else micro
    if cfg.batch % M:
        raise ValueError("mini-batch must split into M equal micro-batches")
    c = gp.gp_config()
    c.seq_len = cfg.seq
    c.seqs_per_microbatch = cfg.batch // M
    c.num_microbatches = M
    c.dtype = DTYPES[cfg.dtype][0]
    c.kind = KINDS[cfg.kind]
    c.mem_seq_len = cfg.mem_seq
    c.loss = LOSSES[cfg.loss]
    c.vocab = cfg.vocab
    c.label_smoothing = cfg.label_smoothing
    c.ln_eps = cfg.ln_eps
    c.check_finite = 1 if check_finite else 0
    c.keep_activations = 1 if keep_activations else 0
    c.optimizer = OPTIMIZERS[cfg.optimizer]
    if cfg.optimizer == "rmsprop":
        c.rms_decay = cfg.rms_decay
        c.rms_eps = cfg.rms_eps
    c.logit_clip = cfg.logit_clip
    if cfg.optimizer == "adamw":
        c.adam_beta1, c.adam_beta2, c.adam_eps = cfg.adam_beta1, cfg.adam_beta2, cfg.adam_eps
        c.weight_decay, c.max_grad_norm = cfg.weight_decay, cfg.max_grad_norm
    return c


class Partition:
    """One configured partition on the current HIP device."""

    def __init__(self, cfg, micro: Optional[int] = None, check_finite: bool = False,
                 keep_activations: bool = False):
        self.cfg = cfg
        self.M = cfg.micro if micro is None else micro
        self.tdtype = DTYPES[cfg.dtype][1]
        self._lane = None  # second stream for the odd micro-batches
        self.h = gp.gp_partition_create(cfg.layers, cfg.d_model, cfg.d_ff, cfg.heads)
        try:
            gp.gp_partition_configure(self.h, make_config(cfg, self.M, check_finite, keep_activations))
        except Exception:
            gp.gp_partition_destroy(self.h)
            raise
        self.device = torch.device("cuda", torch.cuda.current_device())

    def close(self):
        if self.h is not None:
            gp.gp_partition_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # -------------------------------------------------------------- params
    def load_params(self, layers: List[Dict[str, np.ndarray]], head: Dict[str, np.ndarray]):
        for l, p in enumerate(layers):
            for name, arr in p.items():
                gp.gp_set_param(self.h, l, gp.PARAM_ID[name], np.ascontiguousarray(arr, dtype=np.float32))
        for name, arr in head.items():
            gp.gp_set_param(self.h, -1, gp.PARAM_ID[name], np.ascontiguousarray(arr, dtype=np.float32))

    def _read(self, fn, shapes_layers, shapes_head):
        layers = []
        for l in range(self.cfg.layers):
            d = {}
            for name, shp in shapes_layers.items():
                a = np.empty(shp, dtype=np.float32)
                fn(self.h, l, gp.PARAM_ID[name], a)
                d[name] = a
            layers.append(d)
        head = {}
        for name, shp in shapes_head.items():
            a = np.empty(shp, dtype=np.float32)
            fn(self.h, -1, gp.PARAM_ID[name], a)
            head[name] = a
        return layers, head

    def grads(self):
        return self._read(gp.gp_get_grad, self.cfg.param_shapes(), self.cfg.head_shapes())

    def params(self):
        return self._read(gp.gp_get_param, self.cfg.param_shapes(), self.cfg.head_shapes())

    def optimizer_state(self):
        """AdamW's (updates, first moments, second moments) or RMSProp's (0, None,
        mean squares), each moment a (layers, head) pair like params()."""
        def read(which):
            return self._read(lambda h, l, pid, a: gp.gp_get_moment(h, l, pid, which, a), self.cfg.param_shapes(),
                              self.cfg.head_shapes())
        adamw = self.cfg.optimizer == "adamw"
        return gp.gp_get_updates(self.h) if adamw else 0, read(1) if adamw else None, read(2)

    def load_optimizer_state(self, state):
        """What optimizer_state() gave, of a partition of the same configuration."""
        updates, *moments = state
        for which, pair in enumerate(moments, 1):
            if pair is None:
                continue
            for l, tensors in [*enumerate(pair[0]), (-1, pair[1])]:
                for name, arr in tensors.items():
                    gp.gp_set_moment(self.h, l, gp.PARAM_ID[name], which, np.ascontiguousarray(arr, dtype=np.float32))
        if self.cfg.optimizer == "adamw":
            gp.gp_set_updates(self.h, updates)

    def memory(self):
        return gp.gp_partition_memory(self.h)

    def param_count(self):
        return gp.gp_param_count(self.h)

    # ------------------------------------------------------------ schedule
    def _stream(self, handle):
        """The stream of a raw handle (None: the current one), and a context in which tensors are allocated for it."""
        if handle is None:
            return torch.cuda.current_stream(self.device), torch.cuda.stream(None)
        stream = torch.cuda.ExternalStream(handle, device=self.device)
        return stream, torch.cuda.stream(stream)

    def device_inputs(self, case, device="cuda"):
        """Move a synthetic case's boundary tensors to the device."""
        t = lambda a: torch.tensor(a, dtype=torch.float32).to(device=device, dtype=self.tdtype).contiguous()
        out = {"x": t(case["x"]), "mem": None if case.get("mem") is None else t(case["mem"])}
        if self.cfg.loss == "mse":
            out["dy"] = t(case["target"])
        elif self.cfg.loss == "none":
            out["dy"] = t(case["dy"])
        else:
            out["dy"] = torch.tensor(case["labels"], dtype=torch.int32, device=device).contiguous()
        return out

    def step(self, x, mem, dy, lr=0.0, want_y=True, want_dx=True, want_dmem=True, want_loss=True,
             stream=None, y=None, dx=None, dmem=None, want_recomputed=False, noalloc=False, fwd_streams=2,
             bwd_streams=2, dlogp=None, dentropy=None):
        """One mini-batch through GPipe's schedule.  x/mem/dy: device tensors
        of the whole mini-batch (dim 0 = sequences).  Returns dict(y, dx, dmem,
        loss); with want_recomputed also "y_remat", the partition output as
        each backward call re-materialised it (gp_recomputed_output), in
        mini-batch order.  noalloc: the forwards go through
        gp_forward_microbatch_noalloc.  fwd_streams=2: the odd micro-batches'
        forwards are issued on a second stream, so that consecutive forwards
        run side by side (the library keeps one first-pass slot per parity);
        the launch stream waits for it before the backwards.  bwd_streams=2:
        likewise the odd micro-batches' backwards (the library runs the two
        members of a recompute pair side by side where it has two backward
        lanes, and orders them itself otherwise); the launch stream waits for
        the second stream before the update.  dlogp, dentropy (fp32 [N, S]):
        dy holds tokens, and the backwards go through
        gp_backward_microbatch_weighted with these weights."""
        M = self.M
        main, allocated_for_it = self._stream(stream)
        st = main.cuda_stream
        lanes = [st]
        if (fwd_streams > 1 or bwd_streams > 1) and M > 1 and self._lane is None:
            self._lane = second_stream()
        if fwd_streams > 1 and M > 1:
            self._lane.wait_stream(main)
            lanes.append(self._lane.cuda_stream)
        with allocated_for_it:
            if want_y and y is None:
                y = torch.empty_like(x)
            if want_dx and dx is None:
                dx = torch.empty_like(x)
            if mem is not None and want_dmem and dmem is None:
                dmem = torch.empty_like(mem)
            y_remat = torch.empty_like(x) if want_recomputed else None
        xs = x.chunk(M)
        ms = mem.chunk(M) if mem is not None else [None] * M
        ys = y.chunk(M) if y is not None else [None] * M
        dys = dy.chunk(M)
        weights = None
        if dlogp is not None or dentropy is not None:
            for name, t, kind in (("dy", dy, torch.int32), ("dlogp", dlogp, torch.float32),
                                  ("dentropy", dentropy, torch.float32)):
                if t is not None and (t.dtype != kind or t.shape != dy.shape or not t.is_contiguous()
                                      or t.device != self.device):
                    raise ValueError(f"{name} must be contiguous {kind} of the tokens' shape on {self.device}")
            weights = [[None] * M if w is None else w.chunk(M) for w in (dlogp, dentropy)]
        dxs = dx.chunk(M) if dx is not None else [None] * M
        dms = dmem.chunk(M) if dmem is not None else [None] * M
        ptr = lambda t: None if t is None else t.data_ptr()
        fwd = gp.gp_forward_microbatch_noalloc if noalloc else gp.gp_forward_microbatch
        for m in range(M):
            fwd(self.h, m, ptr(xs[m]), ptr(ms[m]), ptr(ys[m]), lanes[m % len(lanes)])
        if len(lanes) > 1:
            main.wait_stream(self._lane)
        yr = y_remat.chunk(M) if want_recomputed else None
        blanes = [st]
        if bwd_streams > 1 and M > 1:
            self._lane.wait_stream(main)
            blanes.append(self._lane.cuda_stream)
        for m in range(M - 1, -1, -1):
            bs = blanes[m % len(blanes)]
            if weights is None:
                gp.gp_backward_microbatch_remat(self.h, m, ptr(dys[m]), ptr(dxs[m]), ptr(dms[m]), bs)
            else:
                gp.gp_backward_microbatch_weighted(self.h, m, ptr(dys[m]), *(ptr(w[m]) for w in weights), ptr(dxs[m]),
                                                   ptr(dms[m]), bs)
            if want_recomputed:
                gp.gp_recomputed_output(self.h, ptr(yr[m]), bs)
        if len(blanes) > 1:
            main.wait_stream(self._lane)
        loss = gp.gp_accumulate_and_step(self.h, lr, want_loss, st)
        out = {"y": y, "dx": dx, "dmem": dmem, "loss": loss}
        if want_recomputed:
            out["y_remat"] = y_remat
        return out

    def capture_step(self, x, mem, dy, lr=0.0, dx=None, dmem=None, want_y=False, y=None, dlogp=None, dentropy=None):
        """Capture one whole mini-batch step (M forwards, M backwards, the
        update) into a HIP graph on a capture stream and return it; replay()
        runs the step again on the same buffers, with the same lr.  The capture itself runs no
        work.  The loss is not read (that would synchronise), and the
        partition must not check gradients for finiteness (same reason).
        The step is captured on the capture stream alone (one stream for the
        forwards and the backwards): a capture of the step issued over two
        streams ended in a segmentation fault inside the HIP runtime's end of
        capture, cause not found."""
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.step(x, mem, dy, lr=lr, want_y=want_y, want_dx=dx is not None, want_dmem=dmem is not None,
                      want_loss=False, y=y, dx=dx, dmem=dmem, fwd_streams=1, bwd_streams=1, dlogp=dlogp, dentropy=dentropy)
        return g

    def score(self, x, tokens=None, mem=None, scale=1.0, top=0, stream=None):
        """Log probabilities, entropies and alternatives under the vocabulary
        head (gp_score_sequences) for n S tokens: x [n, S, D] and mem in the
        partition dtype, tokens int32 [n, S].  An ops.TokenLogprobs of rows n S,
        its tensors allocated for `stream` (the current one unless given)."""
        rows = self.cfg.batch // self.M * self.cfg.seq
        if not 0 <= top <= min(gp.GP_TOP_MAX, self.cfg.vocab):
            raise ValueError(f"top must be in [0, min({gp.GP_TOP_MAX}, vocab)]")
        want = {"x": (x, self.tdtype, rows * self.cfg.d_model)}
        if tokens is not None:
            want["tokens"] = (tokens, torch.int32, rows)
        if mem is not None:
            want["mem"] = (mem, self.tdtype, self.cfg.batch // self.M * self.cfg.mem_seq * self.cfg.d_model)
        for name, (t, kind, count) in want.items():
            if t.dtype != kind or t.numel() != count or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"{name} must be contiguous {kind} of {count} elements on {self.device}")
        st, allocated_for_it = self._stream(stream)
        with allocated_for_it:
            logp, lse, entropy = torch.empty((3, rows), dtype=torch.float32, device=self.device).unbind(0)
            top_ids = torch.empty((rows, top), dtype=torch.int32, device=self.device) if top else None
            top_logp = torch.empty((rows, top), dtype=torch.float32, device=self.device) if top else None
        ptr = lambda t: None if t is None else t.data_ptr()
        gp.gp_score_sequences(self.h, x.data_ptr(), ptr(mem), ptr(tokens), scale,
                              logp.data_ptr() if tokens is not None else None, lse.data_ptr(), entropy.data_ptr(), top,
                              ptr(top_ids), ptr(top_logp), st.cuda_stream)
        return TokenLogprobs(logp if tokens is not None else None, lse, entropy, top_ids, top_logp)

    def grad_norm(self):
        """The last step's gradient norm, before clipping (max_grad_norm)."""
        return gp.gp_get_grad_norm(self.h)

    # ------------------------------------------------------------ timers
    def timer_select(self, role):
        """role: a name from gp.KERNEL_ROLES, "all", or None to stop."""
        r = gp.GP_K_NONE if role is None else gp.GP_K_COUNT if role == "all" else gp.KERNEL_ROLE[role]
        gp.gp_timer_select(self.h, r)

    def timer_read(self, role):
        ms, n, flops, nbytes = gp.gp_timer_read(self.h, gp.KERNEL_ROLE[role])
        return {"ms": ms, "launches": n, "flops": flops, "bytes": nbytes}

    def timer_reset(self):
        gp.gp_timer_reset(self.h)

    def timer_sample(self, every):
        """Time one launch in `every` of the selected role (1: all)."""
        gp.gp_timer_sample(self.h, every)
