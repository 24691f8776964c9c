"""GPU: RMMNorm and RMMLinear8 under autograd, the operators one after the other, streams and graphs."""
import pytest
import torch
from torch.autograd import forward_ad

import eight
import paper_2201_13195_amd as rmm

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2


def test_layer_is_the_calls_it_is_made_of():
    torch.manual_seed(0)
    for scale_dtype in eight.SCALES:
        lin = rmm.RMMLinear8(264, 136, rho=0.25, seed=77, layer_id=3, scale_dtype=scale_dtype, grad_f8=E5)
        X = torch.randn(6, 100, 264, device=DEV).bfloat16().requires_grad_(True)
        dY = torch.randn(6, 100, 136, device=DEV).bfloat16()
        Y = lin(X)
        assert Y.shape == (6, 100, 136) and lin.last_state == (77, 3 << 32)
        assert sorted(tuple(t.shape) for t in Y.grad_fn.saved_tensors) == [(136, 264), (150, 264)]      # W and X_proj, not X
        Y.backward(dY)
        X2, dY2, W = X.detach().reshape(-1, 264), dY.reshape(-1, 136), lin.weight.detach()
        w = rmm.rmm_quantize8_weight(W, scale_dtype=scale_dtype, transposed=True)
        assert torch.equal(Y.detach().reshape(-1, 136), rmm.rmm_linear8(*rmm.rmm_quantize8(X2, scale_dtype=scale_dtype), *w[:2], bias=lin.bias.detach()))
        dX = rmm.rmm_linear8(*rmm.rmm_quantize8(dY2, f8=E5, scale_dtype=scale_dtype), *w[2:])
        X_proj = rmm.rmm_sketch(X2, 150, rmm.GAUSSIAN, 77, 3 << 32)
        _, dW, db = rmm.rmm_backward(dY2, W, X_proj, rmm.GAUSSIAN, 77, 3 << 32, need_dX=False, need_dbias=True)
        assert torch.equal(X.grad.reshape(-1, 264), dX) and torch.equal(lin.weight.grad, dW) and torch.equal(lin.bias.grad, db)


def test_the_layer_is_near_the_one_in_bf16():
    """Rounding both operands to 8 bits is off by half a step each, 2^-4 at most of a product's factor; products of both signs add
    up like independent errors, so that the whole is off by less than the sum of the two half steps."""
    torch.manual_seed(1)
    a, b = rmm.RMMLinear(1024, 512, seed=1, layer_id=1), rmm.RMMLinear8(1024, 512, seed=1, layer_id=1)
    b.load_state_dict(a.state_dict())
    X, dY = torch.randn(700, 1024, device=DEV).bfloat16(), torch.randn(700, 512, device=DEV).bfloat16()
    got = []
    for m in (a, b):
        x = X.clone().requires_grad_(True)
        y = m(x)
        y.backward(dY)
        got.append((y.detach().double(), x.grad.double(), m.weight.grad.double(), m.bias.grad.double()))
    for i in (0, 1):
        assert float((got[0][i] - got[1][i]).norm() / got[0][i].norm()) < 2 * 2.0 ** -4
    rel = float((got[0][2] - got[1][2]).norm() / got[0][2].norm())
    assert rel < 2 * eight.HALF[torch.bfloat16]                     # the sketched gradient is the same estimate
    assert float((got[0][3] - got[1][3]).norm() / got[0][3].norm()) < 2 * eight.HALF[torch.bfloat16]


def formula(h, w, dy, dh):
    r = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6)
    hat, g = h * r, dy * w
    return r * (g - hat * (g * hat).mean(-1, keepdim=True)) + dh, (dy * hat).reshape(-1, h.shape[-1]).sum(0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_module_gradients(dtype):
    torch.manual_seed(2)
    norm = rmm.RMMNorm(200, dtype=dtype)
    with torch.no_grad():
        norm.weight.add_(0.1 * torch.randn(200, device=DEV))
    X, R = (torch.randn(4, 33, 200, device=DEV).to(dtype).requires_grad_(True) for _ in range(2))
    dY, dH = torch.randn(4, 33, 200, device=DEV).to(dtype), torch.randn(4, 33, 200, device=DEV).to(dtype)
    tol = 2 * eight.HALF[dtype] + 64 * 2.0 ** -24
    Y, H = norm(X, R)
    torch.autograd.backward([Y, H], [dY, dH])
    dx, dw = formula(H.detach().double(), norm.weight.detach().double(), dY.double(), dH.double())
    for got, want in ((X.grad, dx), (R.grad, dx), (norm.weight.grad, dw)):
        assert float((got.double() - want).norm() / want.norm()) < tol
    # H alone used, Y alone used, without a residual
    X.grad = R.grad = norm.weight.grad = None
    Y, H = norm(X, R)
    H.backward(dH)
    assert torch.equal(X.grad, dH) and torch.equal(R.grad, dH) and norm.weight.grad is None
    X.grad = None
    Y = norm(X)
    Y.backward(dY)
    dx, dw = formula(X.detach().double(), norm.weight.detach().double(), dY.double(), 0)
    assert float((X.grad.double() - dx).norm() / dx.norm()) < tol and float((norm.weight.grad.double() - dw).norm() / dw.norm()) < tol


def test_views_and_expanded_inputs():
    """Rows that are not dense, and a residual that is one row for all (its gradient is the sum over the rows)."""
    torch.manual_seed(3)
    norm, lin = rmm.RMMNorm(128, dtype=torch.float32), rmm.RMMLinear8(128, 64, dtype=torch.float32, k=16)
    base = torch.randn(50, 300, device=DEV, requires_grad=True)
    row = torch.randn(1, 128, device=DEV, requires_grad=True)
    Y, H = norm(base[:, 7:135], row.expand(50, 128))
    out = lin(Y.t().contiguous().t())
    dY = torch.randn_like(out)
    (out * dY).sum().backward()
    assert float(base.grad[:, :7].abs().max()) == 0 and float(base.grad[:, 135:].abs().max()) == 0
    assert torch.allclose(row.grad[0], base.grad[:, 7:135].sum(0), rtol=1e-4, atol=1e-5)


def block(norm, lin, X, R):
    rows, H = norm(X, R)
    return lin(rows), H


@pytest.mark.parametrize("n", [1, 24, 700])
def test_norm_and_layer_together(n):
    """The norm's rows go into the layer as they are: in training and in serving, with packed weights and without."""
    torch.manual_seed(4)
    for scale_dtype in eight.SCALES:
        norm = rmm.RMMNorm(384, f8=E4, scale_dtype=scale_dtype)
        lin = rmm.RMMLinear8(384, 520, seed=5, layer_id=9, scale_dtype=scale_dtype)
        X, R = (torch.randn(n, 384, device=DEV).bfloat16().requires_grad_(True) for _ in range(2))
        Y, H = block(norm, lin, X, R)
        dY = torch.randn_like(Y)
        torch.autograd.backward([Y, H], [dY, torch.ones_like(H)])
        r = rmm.rmm_rms_norm(X.detach(), norm.weight.detach(), R.detach(), f8=E4, scale_dtype=scale_dtype)
        w = rmm.rmm_quantize8_weight(lin.weight.detach(), scale_dtype=scale_dtype, transposed=True)
        assert torch.equal(Y.detach(), rmm.rmm_linear8(r.Y8, r.scales, *w[:2], bias=lin.bias.detach())) and torch.equal(H.detach(), r.H)
        d_mid = rmm.rmm_linear8(*rmm.rmm_quantize8(dY, scale_dtype=scale_dtype), *w[2:])
        dX, dw = rmm.rmm_rms_norm_backward(d_mid, r.H, norm.weight.detach(), r.rstd, torch.ones_like(H))
        assert torch.equal(X.grad, dX) and torch.equal(R.grad, dX) and torch.equal(norm.weight.grad, dw)
        assert lin.weight.grad is not None and torch.isfinite(lin.weight.grad.float()).all()
        with torch.no_grad():
            for m in (lin, lin.pack()):
                out, H2 = block(norm, m, X, R)
                assert torch.equal(out, Y.detach()) and torch.equal(H2, H.detach())
            rows, _ = norm(X, R)
            assert rows.Y is None
        with pytest.raises(ValueError):
            lin(rows)                                     # made without gradients, used with them
        with torch.no_grad():
            lin.weight.mul_(2)
            with pytest.raises(RuntimeError):
                lin(X)
            assert torch.isfinite(lin.pack()(X).float()).all()


def test_frozen_weights_and_inputs():
    lin = rmm.RMMLinear8(128, 64, k=8)
    X = torch.randn(20, 128, device=DEV).bfloat16()
    lin(X).sum().backward()                               # no gradient of X is asked for
    assert lin.weight.grad is not None
    lin.weight.requires_grad_(False), lin.bias.requires_grad_(False)
    lin.weight.grad = None
    X.requires_grad_(True)
    lin(X).sum().backward()
    assert X.grad is not None and lin.weight.grad is None


def test_serving_step_in_a_graph_replayed():
    """Norm, layer, norm, layer for one token, captured once, replayed on new inputs with eager work in between."""
    torch.manual_seed(6)
    norms = [rmm.RMMNorm(512, f8=E4, scale_dtype=torch.float8_e8m0fnu) for _ in range(2)]
    lins = [rmm.RMMLinear8(512, 512).pack() for _ in range(2)]
    X, R = torch.randn(1, 512, device=DEV).bfloat16(), torch.randn(1, 512, device=DEV).bfloat16()

    def step():
        with torch.no_grad():
            x, h = X, R
            for norm, lin in zip(norms, lins):
                x, h = block(norm, lin, x, h)
            return x, h

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, h = step()
    for i in range(4):
        X.copy_(torch.randn(1, 512, device=DEV).bfloat16())
        R.copy_(torch.randn(1, 512, device=DEV).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), h.clone()
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_training_step_in_a_graph_replayed():
    """The calls of a training step on buffers that the graph owns."""
    torch.manual_seed(7)
    n, d_in, d_out = 600, 384, 520
    X, R = (torch.randn(n, d_in, device=DEV).bfloat16() for _ in range(2))
    dY, W, g = torch.randn(n, d_out, device=DEV).bfloat16(), torch.randn(d_out, d_in, device=DEV).bfloat16(), torch.ones(d_in, device=DEV).bfloat16()

    def step():
        r = rmm.rmm_rms_norm(X, g, R, f8=E4)
        w = rmm.rmm_quantize8_weight(W, transposed=True)
        Y = rmm.rmm_linear8(r.Y8, r.scales, *w[:2])
        d = rmm.rmm_linear8(*rmm.rmm_quantize8(dY, f8=E5), *w[2:])
        return (Y,) + tuple(rmm.rmm_rms_norm_backward(d, r.H, g, r.rstd))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        X.copy_(torch.randn(n, d_in, device=DEV).bfloat16())
        dY.copy_(torch.randn(n, d_out, device=DEV).bfloat16())
        W.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_two_streams_at_once():
    torch.manual_seed(8)
    X, W = torch.randn(500, 640, device=DEV).bfloat16(), torch.randn(300, 640, device=DEV).bfloat16()
    g = torch.ones(640, device=DEV).bfloat16()

    def chain():
        r = rmm.rmm_rms_norm(X, g, X, f8=E4)
        Y = rmm.rmm_linear8(r.Y8, r.scales, *rmm.rmm_quantize8_weight(W))
        return Y, rmm.rmm_rms_norm_backward(X, r.H, g, r.rstd)[1]

    want = chain()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(chain())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in got for a, b in zip(out, want))


def test_gradients_of_gradients_are_refused():
    norm, layer = rmm.RMMNorm(64), rmm.RMMLinear8(64, 32)
    for f in (norm, layer):
        X = torch.randn(8, 64, device=DEV, dtype=torch.bfloat16, requires_grad=True)
        g, = torch.autograd.grad(f(X).float().square().sum(), X, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiate twice"):
            g.float().sum().backward()


def test_packed_weights_that_changed_are_refused():
    layer = rmm.RMMLinear8(64, 32)
    X = torch.randn(8, 64, device=DEV, dtype=torch.bfloat16)
    with torch.no_grad():
        want = layer(X)
        assert torch.equal(layer.pack()(X), want)
        layer.weight.mul_(2)
        with pytest.raises(RuntimeError, match="has changed"):
            layer(X)
        assert torch.equal(layer.pack()(X), 2 * want)


class Block(torch.nn.Module):
    def __init__(self, norm, lin):
        super().__init__()
        self.norm, self.lin = norm, lin

    def forward(self, X, R):
        return block(self.norm, self.lin, X, R)


@pytest.mark.parametrize("packed", [False, True])
def test_calls_without_gradients_are_traced_and_refuse_tangents(packed):
    lin = rmm.RMMLinear8(64, 24, k=20, seed=3, layer_id=1)
    norm = rmm.RMMNorm(64, f8=E4, scale_dtype=torch.float8_e8m0fnu)
    X, X2, R = (torch.randn(3, 10, 64, device=DEV, dtype=torch.bfloat16) for _ in range(3))
    both = Block(norm, lin)
    with torch.no_grad():
        if packed:
            lin.pack()
        traced = torch.jit.trace(lin, (X,), check_trace=False)
        for x in (X, X2, X2.reshape(5, 6, 64)):
            assert torch.equal(traced(x), lin(x))
        traced = torch.jit.trace(both, (X, R), check_trace=False)
        for x in (X, X2, X2.reshape(5, 6, 64)):
            assert all(torch.equal(a, b) for a, b in zip(traced(x, R.reshape(x.shape)), both(x, R.reshape(x.shape))))
        with forward_ad.dual_level():
            dual = forward_ad.make_dual(X, torch.ones_like(X))
            for call in (lambda: lin(dual), lambda: norm(dual), lambda: both(X, dual)):
                with pytest.raises(NotImplementedError):
                    call()
        for f in (lin, rmm.RMMNorm(64)):
            with pytest.raises(RuntimeError):
                torch.vmap(f)(X)
    assert lin.calls == 0


def test_tracing_records_the_norm_and_the_layer():
    """With gradients too, as the layer in bf16 does."""
    lin = rmm.RMMLinear8(64, 24, k=20, seed=3, layer_id=1)
    both = Block(rmm.RMMNorm(64, f8=E4, scale_dtype=torch.float8_e8m0fnu), lin)
    X, X2, R = (torch.randn(30, 64, device=DEV, dtype=torch.bfloat16) for _ in range(3))
    traced = torch.jit.trace(both, (X, R), check_trace=False)
    for x in (X, X2):
        lin.calls = 0
        params = (both.norm.weight, lin.weight, lin.bias)
        got, want = traced(x, R), both(x, R)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for a, b in zip(*(torch.autograd.grad(y.float().sum() + h.float().sum(), params) for y, h in (got, want))):
            assert torch.equal(a, b)


def test_slices_and_gradients_that_start_anywhere():
    """Rows of odd widths: a slice, and the gradient that the backward pass of a cat hands on, start off the library's 16 bytes."""
    torch.manual_seed(9)
    for m, d in ((rmm.RMMNorm(1001, dtype=torch.float32), 1001), (rmm.RMMLinear8(1001, 77, k=2, dtype=torch.float32), 77)):
        whole, dY = torch.randn(7, 1001, device=DEV, requires_grad=True), torch.randn(7, d, device=DEV)
        assert whole[3:].data_ptr() % 16 and (3 * d * 4) % 16
        m.calls = 0                                       # (the same sketches both times)
        y = torch.cat([m(whole[:3]), m(whole[3:])])
        got = torch.autograd.grad(y, [whole, m.weight], dY)
        m.calls = 0
        ya, yb = m(whole[:3].clone()), m(whole[3:].clone())
        want = torch.autograd.grad([ya, yb], [whole, m.weight], [dY[:3].clone(), dY[3:].clone()])
        assert torch.equal(y, torch.cat([ya, yb])) and all(torch.equal(a, b) for a, b in zip(got, want))
        with torch.no_grad():
            assert torch.equal(m(whole[3:]), yb)
