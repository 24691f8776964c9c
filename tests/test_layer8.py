"""CPU: RMMNorm and RMMLinear8 as modules, with stand-ins for the calls of the binding: plain numpy, so that neither a trace nor autograd
sees into them, as with the kernels."""
import copy
import io

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


def take(*tensors):
    """What the library checks of its operands."""
    for t in tensors:
        if t is not None and (not t.is_contiguous() or t.data_ptr() % 16):
            raise binding.RmmError(-1, "stand-in")


@pytest.fixture
def stand_ins(monkeypatch):
    """Rows and weights stay what they are, scales are ones; the calls made so far, by name."""
    calls = []

    def quantize8(A, f8=E4, scale_dtype=torch.float32):
        calls.append("quantize8")
        take(A)
        return opaque(number(A).copy()), torch.ones(binding._blocks8(A.shape[1]), A.shape[0]).to(scale_dtype)

    def quantize8_weight(W, f8=E4, scale_dtype=torch.float32, transposed=False):
        calls.append("quantize8_weight")
        take(W)
        scales = torch.ones(binding._blocks8(W.shape[0]), binding._blocks8(W.shape[1])).to(scale_dtype)
        return (opaque(number(W).copy()), scales) + ((opaque(number(W).T.copy()), scales.t()) if transposed else ())

    def linear8(X8, x_scales, W8, w_scales, bias=None, dtype=torch.bfloat16, Y=None):
        calls.append("linear8")
        take(bias)
        return opaque(number(X8) @ number(W8).T + (0 if bias is None else number(bias))).to(dtype)

    def sketch(A, k, kind, seed, offset):
        calls.append("sketch")
        take(A)
        return opaque(number(A)[:k].copy()).to(A.dtype)

    def rms_norm(X, weight, residual=None, eps=1e-6, need_Y=True, f8=None, scale_dtype=torch.float32):
        calls.append("rms_norm")
        take(X, weight, residual)
        h = number(X) + (0 if residual is None else number(residual))
        rstd = 1 / np.sqrt((h * h).mean(1) + eps)
        y = h * rstd[:, None] * number(weight)
        rows = quantize8(opaque(y), f8, scale_dtype) if f8 is not None else (None, None)
        return binding.RMSNormResult(opaque(y).to(X.dtype) if need_Y else None, X if residual is None else opaque(h).to(X.dtype), opaque(rstd), *rows)

    def rms_norm_backward(dY, H, weight, rstd, dH=None, need_dX=True, need_dweight=True):
        calls.append("rms_norm_backward")
        take(dY, H, weight, dH)
        r = rstd[:, None].double()
        g, hat = dY.double() * weight.double(), H.double() * r
        dX = r * (g - hat * (g * hat).mean(1, keepdim=True)) + (0 if dH is None else dH)
        return dX.to(H.dtype), (dY * hat).sum(0).to(H.dtype)

    def backward(dY, W, X_proj, kind, seed, offset, need_dX=True, need_dbias=False):
        calls.append("backward")
        take(dY, W, X_proj)
        return None, opaque(number(dY)[:X_proj.shape[0]].T @ number(X_proj)), opaque(number(dY).sum(0))

    for name, f in (("rmm_quantize8", quantize8), ("rmm_quantize8_weight", quantize8_weight), ("rmm_linear8", linear8), ("rmm_sketch", sketch),
                    ("rmm_rms_norm", rms_norm), ("rmm_rms_norm_backward", rms_norm_backward), ("rmm_backward", backward)):
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


def off_16(*shape):
    """A dense tensor that starts 4 bytes behind a multiple of 16."""
    n = int(np.prod(shape))
    t = torch.randn(n + 1)[1:].view(*shape)
    assert t.is_contiguous() and t.data_ptr() % 16 == 4
    return t


def test_tensors_that_start_anywhere(stand_ins):
    """Slices of rows of odd width are dense and start off the library's 16 bytes; a cat's backward hands such a gradient on."""
    norm = rmm.RMMNorm(15, device="cpu", dtype=torch.float32)
    lin = rmm.RMMLinear8(15, 13, device="cpu", dtype=torch.float32, k=4)
    for m, d in ((norm, 15), (lin, 13)):
        whole = torch.randn(7, 15, requires_grad=True)
        a, b = whole[:3], whole[3:]
        assert b.is_contiguous() and b.data_ptr() % 16
        dY = torch.randn(7, d)
        y = torch.cat([m(a), m(b)])
        y.backward(dY)
        grad, whole.grad = whole.grad, None
        ya, yb = m(whole[:3].clone()), m(whole[3:].clone())
        assert torch.equal(y, torch.cat([ya, yb]))
        torch.autograd.backward([ya, yb], [dY[:3].clone(), dY[3:].clone()])
        assert torch.equal(whole.grad, grad)
        with torch.no_grad():
            assert torch.equal(m(off_16(5, 15).copy_(whole[:5])), m(whole[:5].clone()))
    X, R, dH = off_16(5, 15).requires_grad_(True), off_16(5, 15), off_16(5, 15)
    Y, H = norm(X, R)
    torch.autograd.backward([Y, H], [off_16(5, 15), dH])
    assert X.grad.shape == X.shape


def test_parameters_that_start_anywhere(stand_ins):
    """Views into one flat tensor, as sharding programs make them of parameters."""
    norm = rmm.RMMNorm(16, device="cpu", dtype=torch.float32)
    lin = layer()
    X = torch.randn(5, 16)
    want = lin(norm(X)).detach()
    norm.weight.data = off_16(16).copy_(norm.weight.data)
    lin.weight.data, lin.bias.data = off_16(12, 16).copy_(lin.weight.data), off_16(12).copy_(lin.bias.data)
    out = lin(norm(X))
    out.sum().backward()
    assert torch.equal(out, want) and lin.weight.grad is not None and norm.weight.grad is not None
    with torch.no_grad():
        assert torch.equal(lin(norm(X)), want) and torch.equal(lin.pack()(norm(X)), want)


def test_defaults_of_the_two_modules_fit_together(stand_ins):
    norm, lin = rmm.RMMNorm(16, f8=E4, device="cpu", dtype=torch.float32), layer()
    assert norm.scale_dtype == lin.scale_dtype
    assert torch.isfinite(lin(norm(torch.randn(5, 16)))).all()


@pytest.mark.parametrize("gradients", [False, True])
def test_rows_with_another_kind_of_scales_are_refused_before_anything_happens(stand_ins, gradients):
    norm, lin = rmm.RMMNorm(16, f8=E4, scale_dtype=torch.float32, device="cpu", dtype=torch.float32), layer()
    with torch.set_grad_enabled(gradients):
        rows = norm(torch.randn(5, 16))
        del stand_ins[:]
        with pytest.raises(TypeError, match="scale_dtype"):
            lin(rows)
    assert lin.calls == 0 and not stand_ins


def test_copies_of_a_packed_layer_answer(stand_ins):
    """A copy's weight counts its changes from zero: the packed form stays with the layer that made it."""
    lin, X = layer(), torch.randn(5, 16)
    with torch.no_grad():
        want = lin.pack()(X)
        file = io.BytesIO()
        torch.save(lin, file)
        file.seek(0)
        for other in (copy.deepcopy(lin), copy.copy(lin), torch.load(file, weights_only=False)):
            assert torch.equal(other(X), want)
            other.weight.mul_(2), other.bias.zero_()
            assert torch.equal(other.pack()(X), other(X))


def test_a_training_step_ends_the_packed_form(stand_ins):
    """The fused optimizers change weights without counting it: after a forward pass that trains the weight nothing is answered from before."""
    lin, X = layer(), torch.randn(5, 16)
    opt = torch.optim.AdamW(lin.parameters(), lr=0.1, fused=True)
    with torch.no_grad():
        before = lin.pack()(X)
    lin(X).sum().backward()
    opt.step()
    with torch.no_grad():
        after = lin(X)
        assert not torch.equal(after, before) and torch.allclose(after, X @ lin.weight.t() + lin.bias, atol=1e-5)
        assert torch.equal(lin.pack()(X), after)
    lin.weight.requires_grad_(False)
    lin(X).sum().backward()
    del stand_ins[:]
    with torch.no_grad():
        lin(X)
    assert "quantize8_weight" not in stand_ins              # (a frozen weight stays packed)


def test_a_packed_form_that_ends_under_a_call(stand_ins):
    """Another thread's training call may end it at any moment: a call that has begun goes on with what it has read."""
    class Ends(rmm.RMMLinear8):
        def __getattribute__(self, name):
            value = super().__getattribute__(name)
            if name == "_packed" and value is not None:
                self.__dict__["_packed"] = None             # as if by another thread, right behind the read
            return value

    lin, X = layer(), torch.randn(5, 16)
    with torch.no_grad():
        want = lin.pack()(X)
        lin.__class__ = Ends
        assert torch.equal(lin(X), want) and torch.equal(lin(X), want)
