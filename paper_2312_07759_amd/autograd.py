"""torch.autograd front end of the quantisation layer W -> r_tau(W, C*(W)) (Alg. 2, per-layer steps), of products with
layers in their stored form or in 8-bit integers, of lookups in embedding tables and of the loss against the unquantised network.

Argument marshalling only: the quantisation's forward is one idkm_forward call, its backward one idkm_backward call on the same
context; every step runs in the library's kernels.  One context per layer (the library keeps C*, n*, F* and a borrowed
pointer to W between the two calls).
"""
from __future__ import annotations

import threading

import torch
from torch.autograd.function import once_differentiable

from . import binding


class _Quantize(torch.autograd.Function):
    @staticmethod
    def forward(fn, W, C0, layer):
        fn.layer = layer
        Z, d = W.detach(), C0.shape[1]
        layer.turn += 1
        fn.turn = layer.turn
        if layer.group:
            S, Z = layer.ctx.group_scale(Z, layer.group)
            layer.S = S
        out = layer.ctx.forward(Z.view(-1, d), C0, layer.tau, layer.tol, layer.max_iter, layer.dist, want_Wq=True)
        layer.last_forward = out["info"]
        layer.C = out["C"]
        Wq = out["Wq"].view(W.shape)
        if layer.group:
            fn.scaled = Z, S, Wq
            Wq = layer.ctx.group_unscale(Wq, S, layer.group)
        fn.mark_non_differentiable(out["C"])
        return Wq, out["C"]

    @staticmethod
    def backward(fn, dWq, _dC):
        layer = fn.layer
        if fn.turn != layer.turn:  # the library's state, W's borrowed address in it, is of that other call
            raise RuntimeError("the layer has been quantised again since: its backward pass has to come first")
        dWq = dWq.contiguous()
        if layer.group:
            Z, S, Zq = fn.scaled
            dWq, dS = layer.ctx.group_unscale_backward(dWq, Zq, S, layer.group)
        res = layer.ctx.backward(dWq.view(-1, layer.C.shape[1]), layer.bwd_mode, tol=layer.bwd_tol, max_iter=layer.bwd_max_iter,
                                 alpha=layer.alpha)
        layer.last_backward = res["info"]
        dW = res["dW"].view(dWq.shape)
        if layer.group:
            dW = layer.ctx.group_scale_backward(Z, S, layer.group, dW, dS)
        return dW, None, None


class SoftKMeansQuantize:
    """One layer's quantiser.  `layer(W, C0)` returns (Wq, C*) with Wq differentiable with respect to W by implicit
    differentiation of the soft k-means fixed point (bwd_mode: binding.BWD_IMPLICIT, BWD_JFB, BWD_DENSE, BWD_GMRES).
    C* is returned detached, to warm-start the next step's C0.  The state that a backward pass needs is the last call's: the backward pass
    of a call comes before the next call, or raises.

    group > 0: W is [rows, cols] with cols a multiple of d, and every group of `group` consecutive weights of a row is divided by its
    root mean square before the clustering and multiplied by it after it; the gradient goes through the scales too.  The codebook
    (and tau) are then those of weights of unit size; the scales are kept in `S`.  A multiple of 32 and of d, or at least cols, gives
    layers that `stored` takes."""

    def __init__(self, tau, dist, tol=1e-6, max_iter=200, bwd_mode=binding.BWD_IMPLICIT, bwd_tol=1e-6,
                 bwd_max_iter=1000, alpha=1.0, device=0, group=0):
        self.ctx = binding.Context(device)
        self.tau, self.dist, self.tol, self.max_iter = float(tau), int(dist), float(tol), int(max_iter)
        self.bwd_mode, self.bwd_tol, self.bwd_max_iter, self.alpha = int(bwd_mode), float(bwd_tol), int(bwd_max_iter), float(alpha)
        self.last_forward = self.last_backward = self.C = self.S = None
        self.group, self.turn = int(group), 0
        if self.group < 0:
            raise ValueError("group must be >= 0")

    def __call__(self, W, C0):
        if self.group:
            if W.dim() != 2 or C0.dim() != 2 or W.shape[1] % C0.shape[1]:
                raise ValueError("W must be [rows, cols] with cols a multiple of d, and C0 [k, d]")
        elif W.dim() != 2 or C0.dim() != 2 or W.shape[1] != C0.shape[1]:
            raise ValueError("W must be [m, d] and C0 [k, d]")
        return _Quantize.apply(W.contiguous(), C0.contiguous(), self)

    @torch.no_grad()
    def stored(self, W, C0, dtype=torch.float32):
        """The [rows, cols] layer W solved from C0 and brought to its stored form, every sub-vector replaced by its closest codeword:
        a binding.CodesLayer with a codebook of `dtype` (that of the activations it will be multiplied with).  Solved in a context of its
        own: a backward pass that is still to come finds its state."""
        if W.dim() != 2 or C0.dim() != 2 or W.shape[1] % C0.shape[1]:
            raise ValueError("W must be [rows, cols] with cols a multiple of d, and C0 [k, d]")
        (rows, cols), (k, d) = W.shape, C0.shape
        if self.group and self.group < cols and (self.group % 32 or self.group % d):
            raise ValueError("a stored group shorter than a row must be a multiple of 32 and of d")
        Z, S = W.detach().contiguous(), None
        ctx = binding.Context(self.ctx.device)
        try:
            if self.group:
                S, Z = ctx.group_scale(Z, self.group)
            out = ctx.forward(Z.view(-1, d), C0.contiguous(), self.tau, self.tol, self.max_iter, self.dist, want_Wq=False, want_assign=True)
            words = ctx.pack_codes(out["assign"], k)
        finally:
            ctx.close()
        return binding.CodesLayer(words, rows, cols, out["C"].to(dtype), S, self.group)

    def close(self):
        self.ctx.close()


_local = threading.local()


def _context(device):
    """This thread's context on a device (a context serves one thread at a time, and the backward pass runs on another)."""
    held = _local.__dict__.setdefault("contexts", {})
    if device not in held:
        if torch.cuda.is_current_stream_capturing():  # a context allocates, which would end the capture
            raise RuntimeError("a thread's first call on a device cannot be captured: make one before, or a CodesLinear")
        held[device] = binding.Context(device)
    return held[device]


def _no_capture(*tensors):
    # A graph that records the backward pass of leaves which an eager graph holds too ends the process.
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors) and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("a differentiable call cannot be captured: capture the methods of Context (codes_linear, codes_linear_backward, distill ..)")


def _no_captured_backward():
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("a backward pass cannot be captured: capture Context.codes_linear_backward and distill")


class _CodesProduct(torch.autograd.Function):
    @staticmethod
    def forward(fn, X, C, S, layer, keep8=False):
        ctx, (_, need_C, need_S) = _context(X.get_device()), fn.needs_input_grad[:3]
        fn.layer, fn.kept = layer, None
        held = (X, None)
        if keep8:
            held = (None, None)  # dX does not need X
            if need_C or need_S:
                fn.kept = X.dtype
                kept = ctx.keep8(X)
                held = (kept.Q, kept.E)
        fn.save_for_backward(*held, C, S, layer.words)
        return ctx.codes_linear(layer, X)

    @staticmethod
    @once_differentiable
    def backward(fn, dY):
        _no_captured_backward()
        X, E, C, S, _ = fn.saved_tensors
        need_X, need_C, need_S = fn.needs_input_grad[:3]
        if fn.kept is not None:
            X = binding.Kept8(X, E, fn.layer.cols, fn.kept)
        r = _context(fn.layer.device).codes_linear_backward(fn.layer, X, dY.contiguous(), want_dX=need_X, want_dC=need_C,
                                                            want_dS=need_S)
        return r.get("dX"), r["dC"].to(C.dtype) if need_C else None, r["dS"].to(S.dtype) if need_S else None, None, None


def _as_rows(t):
    """A matrix as the kernels take it, its rows contiguous and apart: itself, or a copy (of a transposed or repeated one, say)."""
    n, width = t.shape
    if (width > 1 and t.stride(1) != 1) or (n > 1 and t.stride(0) < width):
        return t.contiguous()
    return t


class CodesLinear(torch.nn.Module):
    """Product with a [rows, cols] layer in its stored form (binding.CodesLayer): X [..., cols] of any strides -> X w^T [..., rows], in X's
    type (float32, float16 or bfloat16).  The codes stay; the codebook C (float32) and the scales S are parameters, so that both, and
    what lies below, can be trained.  keep8: X is kept in 8 bits (binding.Context.keep8) between the forward and the backward pass, a quarter of
    float32's memory and half of 16 bits'; dC and dS are then those of the kept X, dX is the same."""

    def __init__(self, layer, keep8=False):
        super().__init__()
        _context(layer.device)
        self.rows, self.cols, self.group, self.keep8 = layer.rows, layer.cols, layer.group, bool(keep8)
        self.register_buffer("words", layer.words)
        self.C = torch.nn.Parameter(layer.C.detach().to(torch.float32, copy=True))
        self.S = torch.nn.Parameter(layer.S.detach().clone()) if layer.S is not None else None

    def layer(self, dtype, copy=False):
        """The stored layer as it is now, with its codebook in `dtype`.  copy: codebook and scales stay as they are now, also where the
        parameters are written to behind autograd's back (through .data)."""
        S = None if self.S is None else self.S.detach().to(torch.float32, copy=copy).contiguous()
        C = self.C.detach().to(dtype, copy=copy).contiguous()
        return binding.CodesLayer(self.words, self.rows, self.cols, C, S, self.group)

    def forward(self, X):
        if X.shape[-1] != self.cols:
            raise ValueError(f"X must be [..., {self.cols}], got {tuple(X.shape)}")
        _no_capture(X, self.C, self.S)
        tracked = torch.is_grad_enabled() and (X.requires_grad or self.C.requires_grad or (self.S is not None and self.S.requires_grad))
        layer = self.layer(X.dtype, copy=tracked)
        return _CodesProduct.apply(_as_rows(X.reshape(-1, self.cols)), self.C, self.S, layer, self.keep8 and tracked).view(*X.shape[:-1], self.rows)


def _ids(ids):
    if ids.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"ids must be int32 or int64, got {ids.dtype}")
    return ids.reshape(-1).contiguous()


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(fn, W, ids, alpha, dtype):
        fn.rows, fn.alpha = W.shape[0], alpha
        fn.save_for_backward(ids)
        return _context(W.get_device()).embedding(W, ids, alpha, dtype)

    @staticmethod
    @once_differentiable
    def backward(fn, dY):
        _no_captured_backward()
        ids, = fn.saved_tensors
        return _context(ids.get_device()).embedding_backward(_as_rows(dY), ids, fn.rows, fn.alpha), None, None, None


def embedding(ids, W, alpha=1.0, dtype=torch.float32):
    """Rows ids [...] (int32 or int64; a negative one is padding, a row of zeros) of the float32 table W [rows, cols], times alpha, [..., cols] in
    `dtype`; differentiable in W (SoftKMeansQuantize's Wq, say), whose gradient is float32."""
    if W.dim() != 2:
        raise ValueError(f"W must be [rows, cols], got {tuple(W.shape)}")
    _no_capture(W)
    return _Embedding.apply(W.contiguous(), _ids(ids), float(alpha), dtype).view(*ids.shape, W.shape[1])


class _CodesLookup(torch.autograd.Function):
    @staticmethod
    def forward(fn, C, S, ids, layer, alpha):
        fn.layer, fn.alpha = layer, alpha
        fn.save_for_backward(C, S, ids, layer.words)
        return _context(layer.device).codes_embedding(layer, ids, alpha)

    @staticmethod
    @once_differentiable
    def backward(fn, dY):
        _no_captured_backward()
        C, S, ids, _ = fn.saved_tensors
        need_C, need_S = fn.needs_input_grad[:2]
        r = _context(fn.layer.device).codes_embedding_backward(fn.layer, ids, _as_rows(dY), fn.alpha, want_dC=need_C, want_dS=need_S)
        return r["dC"].to(C.dtype) if need_C else None, r["dS"].to(S.dtype) if need_S else None, None, None, None


class CodesEmbedding(torch.nn.Module):
    """Embedding table in its stored form (a [rows, cols] binding.CodesLayer): ids [...] (int32 or int64; a negative one is padding, a row of zeros) ->
    alpha times their rows, [..., cols] in `dtype` (the layer's unless given).  The codes stay; the codebook C (float32) and the scales S are parameters."""

    def __init__(self, layer, alpha=1.0, dtype=None):
        super().__init__()
        _context(layer.device)
        self.rows, self.cols, self.group, self.alpha, self.dtype = layer.rows, layer.cols, layer.group, float(alpha), dtype or layer.dtype
        self.register_buffer("words", layer.words)
        self.C = torch.nn.Parameter(layer.C.detach().to(torch.float32, copy=True))
        self.S = torch.nn.Parameter(layer.S.detach().clone()) if layer.S is not None else None

    layer = CodesLinear.layer

    def forward(self, ids):
        _no_capture(self.C, self.S)
        tracked = torch.is_grad_enabled() and (self.C.requires_grad or (self.S is not None and self.S.requires_grad))
        layer = self.layer(self.dtype, copy=tracked)
        return _CodesLookup.apply(self.C, self.S, _ids(ids), layer, self.alpha).view(*ids.shape, self.cols)


class _Int8Product(torch.autograd.Function):
    @staticmethod
    def forward(fn, X, layer):
        fn.layer = layer
        fn.save_for_backward(layer.W8, layer.scale)
        return _context(X.get_device()).int8_linear(layer, X)

    @staticmethod
    @once_differentiable
    def backward(fn, dY):
        _no_captured_backward()
        _ = fn.saved_tensors  # integers and scales that were changed in place since are refused
        return _context(fn.layer.device).int8_linear_backward(fn.layer, _as_rows(dY)), None


class Int8Linear(torch.nn.Module):
    """Product in 8-bit integers with a layer that stays as it is (binding.Int8Layer, see binding.Context.int8_layer): X [..., cols] of any strides ->
    [..., rows], in X's type (float32, float16 or bfloat16).  X's rows are brought to integers in the call; the gradient in X is that of
    the product with X itself, so that what lies below can be trained."""

    def __init__(self, layer):
        super().__init__()
        _context(layer.device)
        self.rows, self.cols = layer.rows, layer.cols
        self.register_buffer("W8", layer.W8)
        self.register_buffer("scale", layer.scale)

    def layer(self, dtype):
        """The layer as it is now, for activations of `dtype`."""
        return binding.Int8Layer(self.W8, self.scale.float(), dtype, self.cols)

    def forward(self, X):
        if X.shape[-1] != self.cols:
            raise ValueError(f"X must be [..., {self.cols}], got {tuple(X.shape)}")
        _no_capture(X)
        return _Int8Product.apply(_as_rows(X.reshape(-1, self.cols)), self.layer(X.dtype)).view(*X.shape[:-1], self.rows)


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(fn, logits, index, teacher, tau):
        fn.tau = tau
        fn.save_for_backward(logits, index, teacher)
        return _context(logits.get_device()).distill(logits, index, teacher, tau)[0]

    @staticmethod
    @once_differentiable
    def backward(fn, dloss):
        _no_captured_backward()
        logits, index, teacher = fn.saved_tensors
        return _context(logits.get_device()).distill(logits, index, teacher, fn.tau, dloss.float().contiguous())[2], None, None, None


def distill(logits, index, teacher, tau=1.0):
    """Losses [n] of logits [n, V] (any strides) against the teacher's largest logits (index int32, teacher float32, both [n, top]; a negative index is no
    entry; see binding.Context.distill), differentiable in the logits."""
    _no_capture(logits)
    if logits.dim() == 2:
        logits = _as_rows(logits)
    return _Distill.apply(logits, index, teacher, float(tau))
