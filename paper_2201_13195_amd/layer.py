"""Drop-in layer over the C ABI: `torch.autograd.Function` + `nn.Module` form of Algorithm 1
(the paper's user-facing form, Section 3: a linear layer whose backward uses the sketched input).

Argument marshalling only: the forward is one `rmm_forward` call, the backward one
`rmm_backward` call; autograd keeps X_proj and the 16-byte sketch state, not X (Section 2.4.1).
Both run in the native module (binding.host()) where it takes the arguments: its autograd node
costs a fraction of a Python function's.
"""
import itertools
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding

_layer_ids = itertools.count()     # process-wide: layers built without an explicit layer_id get distinct ones


class RMMLinearFunction(torch.autograd.Function):
    """Y = X W^T (+ b); backward: dX = dY W exactly, dW = (S^T dY)^T (S^T X), db = dY^T 1."""

    @classmethod
    def apply(cls, X, W, bias, k, kind, seed, offset):
        Y = binding._native("linear", X, W, bias, k, kind, seed, offset)
        return super().apply(X, W, bias, k, kind, seed, offset) if Y is None else Y

    @staticmethod
    def forward(ctx, X, W, bias, k, kind, seed, offset):
        lead = X.shape[:-1]
        X2 = X.reshape(-1, X.shape[-1])
        if not X2.is_contiguous():
            X2 = X2.contiguous()
        Wc = W if W.is_contiguous() else W.contiguous()
        Y, X_proj = binding.rmm_forward(X2, Wc, bias, k, kind, seed, offset)
        ctx.save_for_backward(Wc, X_proj)          # X itself is not kept
        ctx.state = (kind, seed, offset)
        ctx.lead, ctx.has_bias = lead, bias is not None
        return Y.reshape(*lead, W.shape[0])

    @staticmethod
    def backward(ctx, dY):
        W, X_proj = ctx.saved_tensors
        kind, seed, offset = ctx.state
        dY2 = dY.reshape(-1, dY.shape[-1])
        if not dY2.is_contiguous():
            dY2 = dY2.contiguous()
        dX, dW, db = binding.rmm_backward(dY2, W, X_proj, kind, seed, offset, need_dX=ctx.needs_input_grad[0],
                                          need_dbias=ctx.has_bias and ctx.needs_input_grad[2])
        if dX is not None:
            dX = dX.reshape(*ctx.lead, W.shape[1])
        return dX, dW, db, None, None, None, None


class RMMInferFunction(torch.autograd.Function):
    """Y alone (Eq. 1), as a call that a trace records and that refuses forward-mode tangents."""

    @classmethod
    def apply(cls, X, W, bias, kind):
        Y = binding._native("infer", X, W, bias, kind)
        return super().apply(X, W, bias, kind) if Y is None else Y

    @staticmethod
    def forward(ctx, X, W, bias, kind):
        Y, _ = binding.rmm_forward(X.reshape(-1, X.shape[-1]).contiguous(), W.detach().contiguous(), bias, 1, kind, 0, 0,
                                   need_xproj=False)
        return Y.reshape(*X.shape[:-1], W.shape[0])


class RMMLinear(torch.nn.Module):
    """`nn.Linear` replacement.  The sketch size is `k` tokens, or `round(rho * n)` of the n
    tokens of each call (clamped to [1, n]); every forward call that will be followed by a
    backward call draws a fresh sketch: state (seed, offset = layer_id * 2^32 + call counter), so
    that sketches of different layers and steps are independent of each other and of dY
    (Section 2.1).  `layer_id` defaults to a process-wide running number.  With gradients disabled
    the layer computes Y only: no sketch, no state consumed."""

    def __init__(self, in_features, out_features, bias=True, rho=0.1, k=None, kind=binding.GAUSSIAN, seed=0,
                 layer_id=None, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.in_features, self.out_features = in_features, out_features
        self.rho, self.k, self.kind, self.seed = rho, k, kind, seed
        self.layer_id = next(_layer_ids) if layer_id is None else int(layer_id)
        self.calls = 0
        self.weight = torch.nn.Parameter(torch.empty((out_features, in_features), device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros((out_features,), device=device, dtype=dtype)) if bias else None
        torch.nn.init.normal_(self.weight, std=0.02)

    def sketch_size(self, n):
        k = self.k if self.k is not None else int(self.rho * n + 0.5)
        return max(1, min(int(k), n))

    def next_state(self):
        offset = (self.layer_id << 32) | (self.calls & 0xFFFFFFFF)
        self.__dict__["calls"] = self.calls + 1     # (a plain attribute: no need for Module.__setattr__'s search)
        return self.seed, offset

    def forward(self, X):
        if not torch.is_grad_enabled():        # nothing will be kept for a backward pass: Y alone
            return RMMInferFunction.apply(X, self.weight, self.bias, self.kind)
        n = X.numel() // X.shape[-1]
        seed, offset = self.__dict__["last_state"] = self.next_state()
        return RMMLinearFunction.apply(X, self.weight, self.bias, self.sketch_size(n), self.kind, seed, offset)


# ---- the layer with its plain products in 8 bits, and the norm in front of it


class Rows8(NamedTuple):
    """Activations in 8-bit rows (binding.rmm_quantize8's data and scales), and the same activations in the layer's dtype where
    a backward pass will follow (None without gradients: the sketch is all that reads them)."""
    Y: Optional[torch.Tensor]
    data: torch.Tensor                # n x d
    scales: torch.Tensor
    lead: Tuple[int, ...]             # the leading sizes that the n rows stand for


def _dense(t):
    """t (or None) as the library takes it: contiguous, from a multiple of 16 bytes on.  (A slice of rows of odd width, which the backward
    pass of a cat hands on too, or a parameter in a flat one may be contiguous and start anywhere.)"""
    if t is None:
        return None
    if not t.is_contiguous():
        t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _rows(X):
    return None if X is None else _dense(X.reshape(-1, X.shape[-1]))


class RMMNormFunction(torch.autograd.Function):
    """(Y, H, Y8, scales) of binding.rmm_rms_norm; gradients of X, residual and weight from those of Y and H."""

    @staticmethod
    def forward(ctx, X, residual, weight, eps, f8, scale_dtype, need_Y):
        r = binding.rmm_rms_norm(_rows(X), _dense(weight), _rows(residual), eps, need_Y, f8, scale_dtype)
        ctx.set_materialize_grads(False)
        H = X if residual is None else r.H.reshape(X.shape)
        ctx.save_for_backward(H, weight, r.rstd)
        ctx.has_residual = residual is not None
        if r.Y8 is not None:
            ctx.mark_non_differentiable(r.Y8, r.scales)
        return None if r.Y is None else r.Y.reshape(X.shape), None if residual is None else H, r.Y8, r.scales

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY, dH, _, __):
        H, weight, rstd = ctx.saved_tensors
        dX, dweight = dH, None
        if dY is not None:
            need_dX, need_dw = ctx.needs_input_grad[0] or ctx.needs_input_grad[1], ctx.needs_input_grad[2]
            if need_dX or need_dw:
                dX, dweight = binding.rmm_rms_norm_backward(_rows(dY), _rows(H), _dense(weight), rstd, _rows(dH), need_dX, need_dw)
            dX = None if dX is None else dX.reshape(H.shape)
        return dX, dX if ctx.has_residual else None, dweight, None, None, None, None


class RMMNorm(torch.nn.Module):
    """Root-mean-square norm over the last dimension: Y = H / sqrt(mean H^2 + eps) * weight, H = X (+ residual).
    `norm(X)` returns Y, `norm(X, residual)` returns (Y, H).  With `f8` (a float8 dtype) Y comes as Rows8, which RMMLinear8 takes
    as it is (both have powers of two as their default scales): the 8-bit rows cost no pass of their own."""

    def __init__(self, features, eps=1e-6, f8=None, scale_dtype=torch.float8_e8m0fnu, device="cuda", dtype=torch.bfloat16):
        super().__init__()
        self.eps, self.f8, self.scale_dtype = float(eps), f8, scale_dtype
        self.weight = torch.nn.Parameter(torch.ones((features,), device=device, dtype=dtype))

    def forward(self, X, residual=None):
        if residual is not None and residual.shape != X.shape:
            raise ValueError("residual must have the shape of X, %s, has %s" % (tuple(X.shape), tuple(residual.shape)))
        need_Y = self.f8 is None or torch.is_grad_enabled()
        Y, H, Y8, scales = RMMNormFunction.apply(X, residual, self.weight, self.eps, self.f8, self.scale_dtype, need_Y)
        if self.f8 is not None:
            Y = Rows8(Y, Y8, scales, tuple(X.shape[:-1]))
        return Y if residual is None else (Y, H)


class RMMLinear8Function(torch.autograd.Function):
    """Y = X8 W8^T (+ b); backward: dX = dY8 W8, dW = (S^T dY)^T (S^T X) from X and dY before they are rounded, db = dY^T 1.
    The roundings to 8 bits have derivative one.  Kept for the backward pass: W and X_proj, as in RMMLinearFunction; the 8-bit
    weights are made again there (they would be as much memory as the saved activations)."""

    @staticmethod
    def forward(ctx, X, data, scales, W, bias, k, kind, seed, offset, scale_dtype, grad_f8):
        X2, Wc = _rows(X), _dense(W)
        if data is None:
            data, scales = binding.rmm_quantize8(X2, scale_dtype=scale_dtype)
        w8, w_scales = binding.rmm_quantize8_weight(Wc, scale_dtype=scale_dtype)
        Y = binding.rmm_linear8(data, scales, w8, w_scales, _dense(bias), X.dtype)
        X_proj = binding.rmm_sketch(X2, k, kind, seed, offset)
        ctx.save_for_backward(Wc, X_proj)
        ctx.state, ctx.formats = (kind, seed, offset), (scale_dtype, grad_f8)
        ctx.lead, ctx.has_bias = X.shape[:-1], bias is not None
        return Y.reshape(*X.shape[:-1], W.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dY):
        W, X_proj = ctx.saved_tensors
        scale_dtype, grad_f8 = ctx.formats
        dY2, dX, dW, db = _rows(dY), None, None, None
        if ctx.needs_input_grad[0]:
            w8 = binding.rmm_quantize8_weight(W, scale_dtype=scale_dtype, transposed=True)
            dX = binding.rmm_linear8(*binding.rmm_quantize8(dY2, f8=grad_f8, scale_dtype=scale_dtype), *w8[2:], None, dY.dtype)
            dX = dX.reshape(*ctx.lead, W.shape[1])
        need_db = ctx.has_bias and ctx.needs_input_grad[4]
        if ctx.needs_input_grad[3] or need_db:
            _, dW, db = binding.rmm_backward(dY2, W, X_proj, *ctx.state, need_dX=False, need_dbias=need_db)
        return (dX, None, None, dW if ctx.needs_input_grad[3] else None, db) + (None,) * 6


class RMMInfer8Function(torch.autograd.Function):
    """RMMLinear8's n x d_out result alone, as a call that a trace records and that refuses forward-mode tangents.  (W: for the tangent
    that it may have, and the parameter of a traced copy.)"""

    @staticmethod
    def forward(ctx, X, data, scales, W, bias, layer):
        return layer._infer(X, data, scales, W, bias)


class RMMLinear8(RMMLinear):
    """RMMLinear with Y and dX as products of 8-bit operands: X, dY in rows with a scale for each 128 columns, W with one for each
    128 x 128 block, made anew from W in every call; the weight gradient is RMMLinear's sketched estimate.  Takes a tensor, or the
    Rows8 of an RMMNorm in front of it.  `scale_dtype`: torch.float32, or torch.float8_e8m0fnu for powers of two;
    `grad_f8`: the format of dY's rows.

    pack() keeps W's 8-bit form for calls without gradients, until W changes: such a call refuses then (what torch does not count goes
    unnoticed: a change through weight.data, or by a fused optimizer).  A forward pass that trains W, as it changes next, ends it; copies
    of the layer, and what .to() makes of it, are not packed."""

    def __init__(self, in_features, out_features, bias=True, rho=0.1, k=None, kind=binding.GAUSSIAN, seed=0, layer_id=None,
                 device="cuda", dtype=torch.bfloat16, scale_dtype=torch.float8_e8m0fnu, grad_f8=torch.float8_e4m3fn):
        super().__init__(in_features, out_features, bias, rho, k, kind, seed, layer_id, device, dtype)
        binding._check_f8(grad_f8, scale_dtype)
        self.scale_dtype, self.grad_f8, self._packed = scale_dtype, grad_f8, None

    def _apply(self, fn, recurse=True):
        self._packed = None
        return super()._apply(fn, recurse)

    def __getstate__(self):
        return {**self.__dict__, "_packed": None}       # (a copy's weight is another, and counts its changes from zero)

    def pack(self):
        W = self.weight.detach()
        self._packed = (binding.rmm_quantize8_weight(_dense(W), scale_dtype=self.scale_dtype), self.weight, self.weight._version)
        return self

    def _weight8(self, W):
        packed = self._packed                    # (once: a training call in another thread may end it)
        if packed is None:
            return binding.rmm_quantize8_weight(_dense(W.detach()), scale_dtype=self.scale_dtype)
        w8, of, version = packed
        if of is not self.weight or version != self.weight._version:
            raise RuntimeError("RMMLinear8: the weight has changed since pack(); call pack() again")
        return w8

    def _infer(self, X, data, scales, W, bias):
        if data is None:
            data, scales = binding.rmm_quantize8(_rows(X), scale_dtype=self.scale_dtype)
        return binding.rmm_linear8(data, scales, *self._weight8(W), _dense(None if bias is None else bias.detach()), W.dtype)

    def forward(self, X):
        rows = X if isinstance(X, Rows8) else None
        if rows is not None and rows.data.shape[1] != self.in_features:
            raise ValueError("RMMLinear8: rows of %d columns, in_features is %d" % (rows.data.shape[1], self.in_features))
        full = X if rows is None else rows.Y
        if full is not None and full.dtype != self.weight.dtype:
            raise TypeError("RMMLinear8: X must have the weight's dtype, %s, has %s" % (self.weight.dtype, full.dtype))
        if rows is not None and rows.scales.dtype != self.scale_dtype:
            raise TypeError("RMMLinear8: rows with scales of %s, the layer's scale_dtype is %s" % (rows.scales.dtype, self.scale_dtype))
        if not torch.is_grad_enabled():
            lead = X.shape[:-1] if rows is None else rows.lead
            args = (X, None, None) if rows is None else (None, rows.data, rows.scales)
            args += (self.weight, self.bias)
            Y = RMMInfer8Function.apply(*args, self) if binding.watched(*args) else self._infer(*args)
            return Y.reshape(*lead, self.out_features)
        if rows is not None:
            if rows.Y is None:
                raise ValueError("RMMLinear8: these rows were made without gradients; a backward pass needs them in the layer's dtype too")
            X, data, scales = rows.Y, rows.data, rows.scales
        else:
            data = scales = None
        if self.weight.requires_grad:
            self.__dict__["_packed"] = None
        n = X.numel() // X.shape[-1]
        seed, offset = self.__dict__["last_state"] = self.next_state()
        return RMMLinear8Function.apply(X, data, scales, self.weight, self.bias, self.sketch_size(n), self.kind, seed, offset,
                                        self.scale_dtype, self.grad_f8)
