"""CPU: refusals of the 8-bit entry points and of their binding, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2201_13195_amd as rmm
from paper_2201_13195_amd import binding

FAKE, ODD = 0x1000, 0x1004                 # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return rmm.load_library()


def mat(data=FAKE, ld=256, scales=FAKE, ld_scales=64, f8=0, scale=0):
    return ctypes.byref(binding._Mat8(data, ld, scales, ld_scales, f8, scale))


BAD = [dict(data=None), dict(data=ODD), dict(scales=None), dict(scales=ODD), dict(ld=240), dict(ld=264), dict(f8=2), dict(f8=-1),
       dict(scale=2), dict(ld=1 << 32)]


def test_quantize8(lib):
    def call(n=64, d=256, dtype=1, A=FAKE, out=None):
        return lib.rmm_quantize8(n, d, dtype, A, mat() if out is None else out, None)
    for bad in (dict(n=0), dict(d=0), dict(n=-3), dict(dtype=2), dict(A=None), dict(A=ODD), dict(n=1 << 31), dict(n=65)):
        assert call(**bad) == -1, bad
    for bad in BAD + [dict(ld_scales=48), dict(ld_scales=72)]:
        assert call(out=mat(**bad)) == -1, bad
    assert lib.rmm_quantize8(64, 256, 1, FAKE, None, None) == -1


def test_quantize8_weight(lib):
    def call(rows=256, cols=256, dtype=0, W=FAKE, out=None, out_t=None):
        return lib.rmm_quantize8_weight(rows, cols, dtype, W, mat() if out is None else out, out_t, None)
    for bad in (dict(rows=0), dict(cols=0), dict(dtype=-1), dict(W=None), dict(W=ODD)):
        assert call(**bad) == -1, bad
    for bad in BAD + [dict(ld_scales=1)]:
        assert call(out=mat(**bad)) == -1 and call(out_t=mat(**bad)) == -1, bad
    assert call(out_t=mat(f8=1)) == -1 and call(out_t=mat(scale=1)) == -1
    assert lib.rmm_quantize8_weight(256, 256, 0, FAKE, None, None, None) == -1


def test_linear8(lib):
    def call(n=64, d_in=256, d_out=256, dtype=1, X=None, W=None, bias=None, Y=FAKE):
        return lib.rmm_linear8(n, d_in, d_out, dtype, mat() if X is None else X, mat() if W is None else W, bias, Y, None)
    for bad in (dict(n=0), dict(d_in=0), dict(d_out=-1), dict(dtype=3), dict(bias=ODD), dict(Y=None), dict(Y=ODD), dict(n=1 << 31)):
        assert call(**bad) == -1, bad
    for bad in BAD:
        assert call(X=mat(**bad)) == -1 and call(W=mat(**bad)) == -1, bad
    assert call(W=mat(f8=1)) == -1                        # weights are e4m3
    assert call(X=mat(scale=1)) == -1 and call(W=mat(scale=1)) == -1
    assert call(X=mat(ld_scales=48)) == -1 and call(W=mat(ld_scales=1)) == -1


def test_norm(lib):
    def call(n=64, d=256, dtype=1, eps=1e-6, X=FAKE, residual=None, weight=FAKE, H=None, Y=FAKE, Y8=None, rstd=None):
        return lib.rmm_rms_norm(n, d, dtype, eps, X, residual, weight, H, Y, Y8, rstd, None)
    for bad in (dict(n=0), dict(d=0), dict(dtype=2), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")), dict(X=None), dict(X=ODD),
                dict(residual=ODD), dict(weight=None), dict(weight=ODD), dict(H=ODD), dict(Y=None), dict(Y=ODD), dict(rstd=ODD)):
        assert call(**bad) == -1, bad
    for bad in BAD + [dict(ld_scales=48), dict(ld_scales=72)]:
        assert call(Y8=mat(**bad)) == -1, bad


def test_norm_backward(lib):
    def call(n=64, d=256, dtype=1, dY=FAKE, dH=None, H=FAKE, weight=FAKE, rstd=FAKE, dX=FAKE, dweight=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return lib.rmm_rms_norm_backward(n, d, dtype, dY, dH, H, weight, rstd, dX, dweight, ws, ws_bytes, None)
    for bad in (dict(n=0), dict(d=0), dict(dtype=2), dict(dY=None), dict(dY=ODD), dict(dH=ODD), dict(H=None), dict(H=ODD), dict(weight=None),
                dict(rstd=None), dict(rstd=ODD), dict(dX=ODD), dict(dweight=ODD), dict(ws=ODD), dict(dX=None, dweight=None)):
        assert call(**bad) == -1, bad
    need = lib.rmm_rms_norm_workspace_bytes(64, 256, 1)
    assert need >= 256 * 4 and call(ws=None) == -3 and call(ws_bytes=need - 1) == -3
    for bad in ((0, 256, 1), (64, 0, 1), (64, 256, 5), (1 << 31, 256, 1)):
        assert lib.rmm_rms_norm_workspace_bytes(*bad) == 0


def test_the_binding_says_what_is_wrong():
    A, f8 = torch.zeros(8, 32), torch.zeros(8, 32, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        rmm.rmm_quantize8(A)
    with pytest.raises(ValueError):
        rmm.rmm_quantize8_weight(A)
    with pytest.raises(TypeError):
        rmm.rmm_quantize8(A, f8=torch.float16)
    with pytest.raises(TypeError):
        rmm.rmm_quantize8(A, scale_dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        rmm.rmm_quantize8(A.half())
    with pytest.raises(ValueError):
        rmm.rmm_linear8(f8, torch.zeros(1, 8), f8, torch.zeros(1, 1))
    with pytest.raises(TypeError):
        rmm.rmm_linear8(f8, torch.zeros(1, 8), f8, torch.zeros(1, 1), dtype=torch.float16)
    with pytest.raises(ValueError):
        rmm.rmm_rms_norm(A, torch.ones(32))
    with pytest.raises(ValueError):
        rmm.rmm_rms_norm_backward(A, A, torch.ones(32), torch.ones(8))


def test_layers_refuse_unknown_formats():
    with pytest.raises(TypeError):
        rmm.RMMLinear8(8, 8, device="cpu", grad_f8=torch.float16)
    with pytest.raises(TypeError):
        rmm.RMMLinear8(8, 8, device="cpu", scale_dtype=torch.float16)


def test_the_layer_refuses_another_dtype_than_its_weights():
    layer = rmm.RMMLinear8(32, 8, device="cpu")
    X = torch.zeros(4, 32)
    rows = rmm.Rows8(X, X.to(torch.float8_e4m3fn), torch.zeros(1, 4), (4,))
    for x in (X, rows):
        with pytest.raises(TypeError, match="the weight's dtype"):
            layer(x)
        with torch.no_grad(), pytest.raises(TypeError, match="the weight's dtype"):
            layer(x)
