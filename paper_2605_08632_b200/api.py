"""Convenience layer over the binding: owns the device buffers of one problem shape.

It allocates outputs and workspaces with torch once, then every call goes straight to the
C entry points.  No arithmetic of the method happens here.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B


def _check(name, t, shape, dtype, device, rows_only=False):
    """Refuses a tensor the kernels would misread: its type, its sizes, its device, its layout.  `rows_only`: the rows may lie
    further apart than they are long."""
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    if t.is_contiguous():
        return
    if not rows_only or t.dim() != 2:
        raise ValueError(f"{name} must be contiguous")
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")


def _on(device, call, *args):
    """The call with `device` current, as the library wants it."""
    if torch.cuda.current_device() == device.index:
        call(*args)
    else:
        with torch.cuda.device(device):
            call(*args)


def _mask(valid):
    """The kernels read one byte per row: a bool mask is the same bytes."""
    return valid.view(torch.uint8) if valid is not None and valid.dtype == torch.bool else valid


def _pitch(t):
    """Row pitch of a 2-D tensor; the stride of a single row means nothing."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _device(device) -> torch.device:
    dev = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if dev.index is None else dev


class CatLoss:
    """Buffers and calls for one (T, d, V, K, dtype) problem on the current CUDA device."""

    def __init__(self, T: int, d: int, V: int, K: int, dtype: torch.dtype = torch.bfloat16,
                 dW_dtype: torch.dtype = torch.float32, slab_mib: int = 0, device: str = "cuda",
                 fixed_decay_gamma: float | None = None):
        if not torch.cuda.is_available():
            raise RuntimeError("CatLoss needs a CUDA device; there is no CPU path")
        code = {torch.bfloat16: B.CAT_BF16, torch.float32: B.CAT_F32}
        self.dtype, self.dW_dtype = dtype, dW_dtype
        if fixed_decay_gamma is None:
            self.shape = B.make_shape(T, d, V, K, code[dtype], code[dW_dtype], slab_mib=slab_mib)
        else:   # the fixed position decay the paper compares CAT with: weight gamma^k
            self.shape = B.make_shape(T, d, V, K, code[dtype], code[dW_dtype], slab_mib=slab_mib,
                                      weight_mode=B.CAT_WEIGHT_FIXED_DECAY, decay_gamma=float(fixed_decay_gamma))
        self.T, self.d, self.V, self.K = T, d, V, K
        dev = torch.device(device)
        nf, nb = B.cat_loss_workspace_bytes(self.shape, 0), B.cat_loss_workspace_bytes(self.shape, 1)
        if nf == 0 or nb == 0:
            raise ValueError("invalid shape for cat_loss")
        self.ws_fwd = torch.empty(nf, dtype=torch.uint8, device=dev)
        self.ws_bwd = torch.empty(nb, dtype=torch.uint8, device=dev)
        self._ws_fused = None
        self._ws_kd = None
        self._ws_captured = []      # workspaces that a captured graph holds, kept when a larger one takes their place
        self._ws_topk = None
        self.loss3 = None
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        self.lse = torch.empty(T, dtype=torch.float32, device=dev)
        self.conf = torch.empty(T, dtype=torch.float32, device=dev)
        self.weight = torch.empty(T, dtype=torch.float32, device=dev)
        self.stats = torch.zeros(32, dtype=torch.uint8, device=dev)
        self.dH = torch.empty(T, d, dtype=dtype, device=dev)
        self.dW = torch.empty(V, d, dtype=dW_dtype, device=dev)

    def forward(self, H, W, labels, valid=None, conf_ext=None):
        B.cat_loss_fwd(self.shape, H, W, labels, valid, conf_ext, self.loss, self.lse, self.conf, self.weight,
                       self.stats, self.ws_fwd)
        return self.loss

    def backward(self, H, W, labels, valid=None, grad_loss=None, accumulate_dW=False):
        B.cat_loss_bwd(self.shape, H, W, labels, valid, self.lse, self.weight, grad_loss, self.dH, self.dW,
                       accumulate_dW, self.ws_bwd)
        return self.dH, self.dW

    def forward_backward(self, H, W, labels, valid=None, conf_ext=None, grad_loss=None, accumulate_dW=False):
        """cat_loss_fwd_bwd: one call, logits kept per row slab instead of recomputed."""
        if self._ws_fused is None:
            n = B.cat_loss_workspace_bytes(self.shape, 2)
            self._ws_fused = torch.empty(n, dtype=torch.uint8, device=self.loss.device)
        B.cat_loss_fwd_bwd(self.shape, H, W, labels, valid, conf_ext, grad_loss, self.loss, self.lse, self.conf,
                           self.weight, self.stats, self.dH, self.dW, accumulate_dW, self._ws_fused)
        return self.loss, self.dH, self.dW

    def forward_backward_timed(self, H, W, labels, valid=None, conf_ext=None, grad_loss=None, accumulate_dW=False):
        """cat_loss_fwd_bwd_events: same results as forward_backward; returns the stage events
        (start, set-up, then per row slab: label reference, logits GEMM, row kernel, slab preparation,
        dH GEMM, dW GEMM; finalize)."""
        if self._ws_fused is None:
            n = B.cat_loss_workspace_bytes(self.shape, 2)
            self._ws_fused = torch.empty(n, dtype=torch.uint8, device=self.loss.device)
        n_slabs = len(B.cat_loss_fused_slabs(self.shape)) - 1
        events = [torch.cuda.Event(enable_timing=True) for _ in range(6 * n_slabs + 3)]
        B.cat_loss_fwd_bwd_events(self.shape, H, W, labels, valid, conf_ext, grad_loss, self.loss, self.lse, self.conf,
                                  self.weight, self.stats, self.dH, self.dW, accumulate_dW, self._ws_fused, events)
        return events

    def accept_len(self) -> torch.Tensor:
        """cat_accept_len: per-block estimate of the expected acceptance length (Eq. 8) from the
        conf / weight of the last forward."""
        out = torch.empty(self.T // self.K, dtype=torch.float32, device=self.loss.device)
        B.cat_accept_len(self.shape, self.conf, self.weight, out)
        return out

    def kd_forward_backward(self, H, W, labels, valid, Ht, Wt, block_start_host, beta, conf_source=B.CAT_CONF_TARGET,
                            conf_ext=None, grad_loss=None, accumulate_dW=False):
        """cat_kd_loss_fwd_bwd: Eq. 12, CAT-weighted cross-entropy + distillation from the target head.
        Returns (loss3, dH, dW) with loss3 = [total, cross-entropy part, distillation part]."""
        desc = B.make_kd_desc(Ht.shape[0], Ht.shape[1], float(beta), conf_source, ldHt=Ht.stride(0), ldWt=Wt.stride(0))
        n = B.cat_kd_workspace_bytes(self.shape, desc, block_start_host)
        if n == 0:
            raise ValueError("invalid problem for cat_kd_loss_fwd_bwd")
        if self._ws_kd is None or self._ws_kd.numel() < n:
            self._ws_kd = torch.empty(n, dtype=torch.uint8, device=self.loss.device)
        if torch.cuda.is_current_stream_capturing() and not any(w is self._ws_kd for w in self._ws_captured):
            self._ws_captured.append(self._ws_kd)
        if self.loss3 is None:
            self.loss3 = torch.zeros(3, dtype=torch.float32, device=self.loss.device)
        B.cat_kd_loss_fwd_bwd(self.shape, desc, H, W, labels, valid, Ht, Wt, block_start_host, conf_ext, grad_loss,
                              self.loss3, self.lse, self.conf, self.weight, self.stats, self.dH, self.dW, accumulate_dW,
                              self._ws_kd)
        return self.loss3, self.dH, self.dW

    def topk_kd_forward_backward(self, H, W, labels, valid, top_ids, top_logp, block_start=None, beta=0.1, renormalize=True,
                                 conf_ext=None, grad_loss=None, accumulate_dW=False):
        """cat_topk_kd_loss_fwd_bwd: Eq. 12 with the distillation term over the teacher's stored top lists `top_ids` [L, k] int64
        and `top_logp` [L, k] fp32 (ids of -1 fill up short lists), as TokenLogProb.forward writes them, in the place of its head.
        Row (block b, position j) reads list block_start[b] + j (int64 [T / K], on the device), or list b * K + j without it.
        renormalize: softmax over the list's entries; otherwise their log probabilities as they are.
        Returns (loss3, dH, dW) with loss3 = [total, cross-entropy part, distillation part]."""
        dev, T, d, V = self.loss.device, self.T, self.d, self.V
        valid = _mask(valid)
        L, k = top_ids.shape
        _check("H", H, (T, d), self.dtype, dev)
        _check("W", W, (V, d), self.dtype, dev)
        _check("labels", labels, (T,), torch.int64, dev)
        _check("top_ids", top_ids, (L, k), torch.int64, dev, rows_only=True)
        _check("top_logp", top_logp, (L, k), torch.float32, dev, rows_only=True)
        if _pitch(top_ids) != _pitch(top_logp):
            raise ValueError("top_ids and top_logp must have the same row pitch")
        for name, t, shape, dtype in (("valid", valid, (T,), torch.uint8), ("block_start", block_start, (T // self.K,), torch.int64),
                                      ("conf_ext", conf_ext, (T,), torch.float32), ("grad_loss", grad_loss, (1,), torch.float32)):
            if t is not None:
                _check(name, t, shape, dtype, dev)
        desc = B.make_topk_kd_desc(L, k, float(beta), renormalize, ld=_pitch(top_ids))
        if not (1 <= k <= B.CAT_TOPK_MAX and L >= 1 and 0.0 <= desc.beta < float("inf")):
            raise ValueError("invalid problem for cat_topk_kd_loss_fwd_bwd")
        if self._ws_topk is None:
            # for lists of any length: a graph captured with one k holds this address while calls with another come and go
            n = B.cat_topk_kd_workspace_bytes(self.shape, B.make_topk_kd_desc(1, B.CAT_TOPK_MAX, 0.0))
            if n == 0:
                raise ValueError("invalid problem for cat_topk_kd_loss_fwd_bwd")
            self._ws_topk = torch.empty(n, dtype=torch.uint8, device=dev)
        if self.loss3 is None:
            self.loss3 = torch.zeros(3, dtype=torch.float32, device=dev)
        _on(dev, B.cat_topk_kd_loss_fwd_bwd, self.shape, desc, H, W, labels, valid, top_ids, top_logp, block_start, conf_ext, grad_loss,
            self.loss3, self.lse, self.conf, self.weight, self.stats, self.dH, self.dW, accumulate_dW, self._ws_topk)
        return self.loss3, self.dH, self.dW

    def topk_kd_status(self) -> int:
        return int(self._ws_topk[:4].view(torch.int32).item())

    def kd_status(self) -> int:
        return int(self._ws_kd[:4].view(torch.int32).item())

    def fused_status(self) -> int:
        return int(self._ws_fused[:4].view(torch.int32).item())

    def bwd_status(self) -> int:
        return int(self.ws_bwd[:4].view(torch.int32).item())

    def fwd_stats(self):
        return B.read_stats(self.stats)


class TargetConfidence:
    """Buffers and calls for cat_conf_fwd / cat_conf_window: target-model confidences of L
    sequence positions (Eq. 9) and their layout as draft rows (Eq. 12)."""

    def __init__(self, L: int, d: int, V: int, dtype: torch.dtype = torch.bfloat16, device: str = "cuda"):
        if not torch.cuda.is_available():
            raise RuntimeError("TargetConfidence needs a CUDA device; there is no CPU path")
        code = {torch.bfloat16: B.CAT_BF16, torch.float32: B.CAT_F32}
        self.L = L
        self.shape = B.make_shape(L, d, V, 1, code[dtype])
        n = B.cat_loss_workspace_bytes(self.shape, 3)
        if n == 0:
            raise ValueError("invalid shape for cat_conf_fwd")
        dev = torch.device(device)
        self.ws = torch.empty(n, dtype=torch.uint8, device=dev)
        self.conf_seq = torch.empty(L, dtype=torch.float32, device=dev)
        self.lse_seq = torch.empty(L, dtype=torch.float32, device=dev)

    def forward(self, Ht, Wt, labels, valid=None):
        B.cat_conf_fwd(self.shape, Ht, Wt, labels, valid, self.conf_seq, self.lse_seq, self.ws)
        return self.conf_seq

    def window(self, block_start: torch.Tensor, K: int) -> torch.Tensor:
        n_blocks = block_start.numel()
        out = torch.empty(n_blocks * K, dtype=torch.float32, device=self.conf_seq.device)
        B.cat_conf_window(self.conf_seq, self.L, block_start, n_blocks, K, out)
        return out

    def status(self) -> int:
        return int(self.ws[:4].view(torch.int32).item())


class LogProbs(NamedTuple):
    """What TokenLogProb.forward returns.  logp is None without labels, top_ids and top_logp without alternatives."""
    logp: torch.Tensor | None        # [T] fp32
    lse: torch.Tensor                # [T] fp32
    entropy: torch.Tensor            # [T] fp32
    top_ids: torch.Tensor | None     # [T, top_k] int64
    top_logp: torch.Tensor | None    # [T, top_k] fp32


class TokenLogProb:
    """Buffers and calls for cat_logprob_fwd / cat_logprob_bwd: log probabilities of given tokens, entropies and the top_k most
    likely tokens of T rows, and the gradients of the first two.  The results are the engine's own buffers: the next
    call overwrites them.  One engine serves one stream at a time."""

    def __init__(self, T: int, d: int, V: int, top_k: int = 0, dtype: torch.dtype = torch.bfloat16,
                 dW_dtype: torch.dtype = torch.float32, slab_mib: int = 0, device: str = "cuda"):
        if not torch.cuda.is_available():
            raise RuntimeError("TokenLogProb needs a CUDA device; there is no CPU path")
        code = {torch.bfloat16: B.CAT_BF16, torch.float32: B.CAT_F32}
        if dtype not in code or dW_dtype not in code:
            raise TypeError("TokenLogProb takes bfloat16 or float32")
        self.T, self.d, self.V, self.top_k, self.dtype, self.dW_dtype, self.slab_mib = T, d, V, top_k, dtype, dW_dtype, slab_mib
        self._code = (code[dtype], code[dW_dtype])
        self._shapes = {}
        n = B.cat_logprob_workspace_bytes(self._shape(d, d), top_k, 0)
        if n == 0:
            raise ValueError("invalid shape for cat_logprob_fwd")
        self.device = _device(device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.ws = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._ws_bwd = self.dH = self.dW = None
        self.logp, self.lse, self.entropy = torch.empty(T, **f32), torch.empty(T, **f32), torch.empty(T, **f32)
        self.top_ids = torch.empty(T, top_k, dtype=torch.int64, device=self.device) if top_k else None
        self.top_logp = torch.empty(T, top_k, **f32) if top_k else None

    def _shape(self, ldH, ldW):
        s = self._shapes.get((ldH, ldW))
        if s is None:
            s = self._shapes[ldH, ldW] = B.make_shape(self.T, self.d, self.V, 1, *self._code, ldH=ldH, ldW=ldW, slab_mib=self.slab_mib)
        return s

    def _inputs(self, H, W, labels, valid):
        _check("H", H, (self.T, self.d), self.dtype, self.device, rows_only=True)
        _check("W", W, (self.V, self.d), self.dtype, self.device, rows_only=True)
        if labels is not None:
            _check("labels", labels, (self.T,), torch.int64, self.device)
        if valid is not None:
            _check("valid", valid, (self.T,), torch.uint8, self.device)

    def forward(self, H, W, labels=None, valid=None) -> LogProbs:
        """Rows of H and W may lie further apart than d (multiples of 8 elements for bfloat16)."""
        valid = _mask(valid)
        self._inputs(H, W, labels, valid)
        logp = None if labels is None else self.logp
        _on(self.device, B.cat_logprob_fwd, self._shape(_pitch(H), _pitch(W)), H, W, labels, valid, self.top_k, logp, self.lse, self.entropy,
            self.top_ids, self.top_logp, self.ws)
        return LogProbs(logp, self.lse, self.entropy, self.top_ids, self.top_logp)

    def backward(self, H, W, labels=None, valid=None, grad_logp=None, grad_entropy=None, lse=None, entropy=None,
                 accumulate_dW=False):
        """(dH, dW) for the upstream gradients of logp and entropy (either may be None).  lse and entropy: those of the forward
        pass on the same rows; the engine's own, of its last forward, unless given."""
        valid = _mask(valid)
        self._inputs(H, W, labels, valid)
        if grad_logp is not None and labels is None:
            raise ValueError("grad_logp needs labels")
        lse = self.lse if lse is None else lse
        entropy = self.entropy if entropy is None else entropy
        for name, t in (("grad_logp", grad_logp), ("grad_entropy", grad_entropy), ("lse", lse), ("entropy", entropy)):
            if t is not None:
                _check(name, t, (self.T,), torch.float32, self.device)
        if _pitch(H) != self.d or _pitch(W) != self.d:
            raise ValueError("backward takes contiguous H and W: the gradients are laid out like them")
        shape = self._shape(self.d, self.d)
        if self._ws_bwd is None:
            n = B.cat_logprob_workspace_bytes(shape, 0, 1)
            self._ws_bwd = torch.empty(n, dtype=torch.uint8, device=self.device)
        if self.dH is None:
            self.dH = torch.empty(self.T, self.d, dtype=self.dtype, device=self.device)
        if self.dW is None:
            if accumulate_dW:
                raise ValueError("accumulate_dW needs a dW to add to: set engine.dW, or run one backward without it")
            self.dW = torch.empty(self.V, self.d, dtype=self.dW_dtype, device=self.device)
        _check("dH", self.dH, (self.T, self.d), self.dtype, self.device)
        _check("dW", self.dW, (self.V, self.d), self.dW_dtype, self.device)
        _on(self.device, B.cat_logprob_bwd, shape, H, W, labels, valid, lse, entropy, grad_logp, grad_entropy, self.dH, self.dW, accumulate_dW,
            self._ws_bwd)
        return self.dH, self.dW

    def status(self) -> int:
        return int(self.ws[:4].view(torch.int32).item())

    def bwd_status(self) -> int:
        return int(self._ws_bwd[:4].view(torch.int32).item())


class _LogProbFn(torch.autograd.Function):
    """autograd glue: cat_logprob_fwd in forward(), cat_logprob_bwd in backward(), through an engine of the call's own.  Its results are the
    caller's; its workspaces go back to torch's allocator as soon as each pass is enqueued, which hands them on in the order of the
    stream."""

    @staticmethod
    def forward(ctx, H, W, labels, valid, engine):
        r = engine.forward(H.detach(), W.detach(), labels, valid)
        engine.ws = engine.logp = engine.lse = engine.entropy = engine.top_ids = engine.top_logp = None
        ctx.engine = engine
        ctx.set_materialize_grads(False)
        # the caller may write to the entropies that are handed out
        ctx.save_for_backward(H, W, labels, valid, r.lse, r.entropy.clone() if any(ctx.needs_input_grad) else r.entropy)
        ctx.mark_non_differentiable(*(t for t in (r.top_ids, r.top_logp) if t is not None))
        return r.logp, r.entropy, r.top_ids, r.top_logp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g_logp, g_entropy, _ids, _tl):
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("LogProbModule's backward pass cannot be captured: capture TokenLogProb.forward and backward")
        H, W, labels, valid, lse, entropy = ctx.saved_tensors
        e = ctx.engine
        dH, dW = e.backward(H.detach(), W.detach(), labels, valid, None if g_logp is None or labels is None else g_logp.contiguous(),
                            None if g_entropy is None else g_entropy.contiguous(), lse=lse, entropy=entropy)
        e.dH = e.dW = e._ws_bwd = None
        return dH, dW, None, None, None


class LogProbModule(torch.nn.Module):
    """Head of a scoring or policy-gradient loop: `logp, entropy, top_ids, top_logp = head(H, labels, valid)` with H [T, d] and
    `weight` [V, d] as the LM head; logp and entropy carry gradients to H and the weight.  The gradient of the weight is formed in
    the weight's type.  Calls share nothing: any lengths, streams and threads.  Not for stream capture with gradients: autograd may then
    wait for other streams inside the capture; capture TokenLogProb.forward and backward instead.  With gradients the weight has to
    be contiguous, and an H whose rows lie further apart is copied."""

    def __init__(self, weight: torch.Tensor, top_k: int = 0, slab_mib: int = 0):
        super().__init__()
        self.weight = weight if isinstance(weight, torch.nn.Parameter) else torch.nn.Parameter(weight)
        self.top_k = top_k
        self.slab_mib = slab_mib

    def forward(self, H, labels=None, valid=None):
        if torch.is_grad_enabled() and (H.requires_grad or self.weight.requires_grad):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("LogProbModule cannot be captured with gradients: capture TokenLogProb.forward and backward")
            if not self.weight.is_contiguous():
                raise ValueError("weight must be contiguous for gradients: theirs are laid out like it")
            H = H.contiguous()
        T, d = H.shape
        engine = TokenLogProb(T, d, self.weight.shape[0], self.top_k, dtype=H.dtype, dW_dtype=self.weight.dtype, slab_mib=self.slab_mib,
                              device=str(H.device))
        return _LogProbFn.apply(H, self.weight, labels, valid, engine)


class _CatLossFn(torch.autograd.Function):
    """autograd glue: the loss and both gradients come out of one cat_loss_fwd_bwd call in forward();
    backward() hands them over, multiplied by the incoming scalar gradient when that is not 1.
    The gradient buffers the call wrote become the graph node's own and the engine gets fresh ones,
    so a second call through the same engine before backward() cannot overwrite them."""

    @staticmethod
    def forward(ctx, H, W, labels, valid, conf_ext, K, engine):
        loss, dH, dW = engine.forward_backward(H.detach(), W.detach(), labels, valid, conf_ext=conf_ext)
        engine.dH, engine.dW = torch.empty_like(dH), torch.empty_like(dW)
        ctx.save_for_backward(dH, dW)
        return loss.clone().reshape(())

    @staticmethod
    def backward(ctx, grad_out):
        dH, dW = ctx.saved_tensors
        if bool((grad_out == 1).item()):
            return dH, dW, None, None, None, None, None
        return dH * grad_out.to(dH.dtype), dW * grad_out.to(dW.dtype), None, None, None, None, None


class CatLossModule(torch.nn.Module):
    """Drop-in loss head for a draft-model training loop: `loss = head(H, labels, valid)` with
    H [T, d] the hidden states of the draft positions (T = blocks * K), using `weight` [V, d] as the
    LM head.  The library's dW is float32; autograd casts it to the parameter's dtype when it stores
    it in `weight.grad`.  An upstream gradient other than 1 is applied by a tensor multiply in
    backward() (chain-rule glue; pass `grad_loss` to CatLoss.forward_backward to have the kernels
    apply a scale instead).  One engine (buffers for one T) is kept per distinct T."""

    def __init__(self, weight: torch.Tensor, K: int, slab_mib: int = 0):
        super().__init__()
        self.weight = weight if isinstance(weight, torch.nn.Parameter) else torch.nn.Parameter(weight)
        self.K = K
        self.slab_mib = slab_mib
        self._engines = {}

    def forward(self, H, labels, valid=None, conf_ext=None):
        T, d = H.shape
        eng = self._engines.get(T)
        if eng is None:
            eng = self._engines[T] = CatLoss(T, d, self.weight.shape[0], self.K, dtype=H.dtype, slab_mib=self.slab_mib,
                                             device=str(H.device))
        return _CatLossFn.apply(H, self.weight, labels, valid, conf_ext, self.K, eng)
