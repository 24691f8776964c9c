"""CPU: RMMNorm and RMMLinear8 as modules, with stand-ins for the calls of the binding: plain numpy, so that neither a trace nor autograd
sees into them, as with the kernels."""
import numpy as np
import pytest
import torch
from torch.autograd import forward_ad

import paper_2201_13195_amd as rmm
from paper_2201_13195_amd import binding

E4 = torch.float8_e4m3fn


def opaque(a):
    return torch.from_numpy(np.ascontiguousarray(a))


def number(t):
    return t.detach().float().numpy()


@pytest.fixture
def stand_ins(monkeypatch):
    """Rows and weights stay what they are, scales are ones; the calls made so far, by name."""
    calls = []

    def quantize8(A, f8=E4, scale_dtype=torch.float32):
        calls.append("quantize8")
        return opaque(number(A).copy()), torch.ones(binding._blocks8(A.shape[1]), A.shape[0]).to(scale_dtype)

    def quantize8_weight(W, f8=E4, scale_dtype=torch.float32, transposed=False):
        calls.append("quantize8_weight")
        scales = torch.ones(binding._blocks8(W.shape[0]), binding._blocks8(W.shape[1])).to(scale_dtype)
        return (opaque(number(W).copy()), scales) + ((opaque(number(W).T.copy()), scales.t()) if transposed else ())

    def linear8(X8, x_scales, W8, w_scales, bias=None, dtype=torch.bfloat16, Y=None):
        calls.append("linear8")
        return opaque(number(X8) @ number(W8).T + (0 if bias is None else number(bias))).to(dtype)

    def sketch(A, k, kind, seed, offset):
        calls.append("sketch")
        return opaque(number(A)[:k].copy()).to(A.dtype)

    def rms_norm(X, weight, residual=None, eps=1e-6, need_Y=True, f8=None, scale_dtype=torch.float32):
        calls.append("rms_norm")
        h = number(X) + (0 if residual is None else number(residual))
        rstd = 1 / np.sqrt((h * h).mean(1) + eps)
        y = h * rstd[:, None] * number(weight)
        rows = quantize8(opaque(y), f8, scale_dtype) if f8 is not None else (None, None)
        return binding.RMSNormResult(opaque(y).to(X.dtype) if need_Y else None, X if residual is None else opaque(h).to(X.dtype), opaque(rstd), *rows)

    for name, f in (("rmm_quantize8", quantize8), ("rmm_quantize8_weight", quantize8_weight), ("rmm_linear8", linear8), ("rmm_sketch", sketch),
                    ("rmm_rms_norm", rms_norm)):
        monkeypatch.setattr(binding, name, f)
    return calls


def layer(**kw):
    torch.manual_seed(1)
    return rmm.RMMLinear8(16, 12, device="cpu", dtype=torch.float32, k=4, **kw)


@pytest.mark.parametrize("packed", [False, True])
def test_calls_without_gradients_are_traced_and_refuse_tangents(stand_ins, packed):
    lin = layer()
    X, X2 = torch.randn(3, 5, 16), torch.randn(3, 5, 16)
    with torch.no_grad():
        if packed:
            lin.pack()
        traced = torch.jit.trace(lin, (X,), check_trace=False)
        for x in (X, X2, torch.randn(2, 9, 16)):
            assert torch.equal(traced(x), lin(x))
        with forward_ad.dual_level(), pytest.raises(NotImplementedError):
            lin(forward_ad.make_dual(X, torch.ones_like(X)))
        with pytest.raises(RuntimeError, match="vmap"):
            torch.vmap(lin)(X)
    assert lin.calls == 0


def test_the_norm_with_the_layer_behind_it_is_traced(stand_ins):
    """The 8-bit rows between them are part of the trace."""
    norm, lin = rmm.RMMNorm(16, f8=E4, scale_dtype=torch.float8_e8m0fnu, device="cpu", dtype=torch.float32), layer()

    class Both(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.norm, self.lin = norm, lin

        def forward(self, X, R):
            rows, H = self.norm(X, R)
            return self.lin(rows), H

    X, R, X2, R2 = (torch.randn(3, 5, 16) for _ in range(4))
    X3, R3 = (torch.randn(2, 9, 16) for _ in range(2))
    both = Both()
    with torch.no_grad():
        traced = torch.jit.trace(both, (X, R), check_trace=False)
        for x, r in ((X, R), (X2, R2), (X3, R3)):
            assert all(torch.equal(a, b) for a, b in zip(traced(x, r), both(x, r)))
        with forward_ad.dual_level(), pytest.raises(NotImplementedError):
            both(forward_ad.make_dual(X, torch.ones_like(X)), R)
        rows, _ = norm(X, R)
        with forward_ad.dual_level(), pytest.raises(NotImplementedError):
            lin(rows._replace(data=forward_ad.make_dual(rows.data, torch.ones_like(rows.data))))
