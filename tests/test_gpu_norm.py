"""GPU: the root-mean-square norm and its backward pass against their formulas in 64 bits.

Sums over d columns: a lane adds at most 8 columns in each of 4 runs (longer rows: d / 1024), ten exchanges and sums of waves follow,
each half a step of fp32; `terms(d)` counts them.  The root halves that of the sum of squares."""
import pytest
import torch

import eight
import paper_2201_13195_amd as rmm

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-6
DTYPES = [torch.bfloat16, torch.float32]
SHAPES = [(1, 1), (1, 1024), (3, 7), (5, 512), (9, 513), (64, 768), (130, 1001), (33, 1024), (17, 1032), (31, 2048), (10, 2049), (6, 4096),
          (7, 5000), (3, 8192), (2, 8200), (2, 20000), (3, 32768), (2, 32776), (3, 50001)]
STEP = 2.0 ** -24


def terms(d):
    return max(32, d // 1024 + 8) + 32


def inputs(n, d, dtype, residual=True, seed=0):
    g = torch.Generator().manual_seed(seed + 31 * n + d)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    size = torch.exp(r(n, 1))
    x = {"X": (r(n, d) * size).to(dtype), "residual": (r(n, d) * size).to(dtype) if residual else None, "weight": (1 + 0.2 * r(d)).to(dtype),
         "dY": r(n, d).to(dtype), "dH": r(n, d).to(dtype)}
    return {k: None if v is None else v.to(DEV) for k, v in x.items()}


def forward64(X, weight, residual, dtype):
    h = X.double() if residual is None else (X.float() + residual.float()).to(dtype).double()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    return h, rstd, h * rstd * weight.double()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", SHAPES)
def test_forward(n, d, dtype, residual):
    t = inputs(n, d, dtype, residual)
    h, rstd, y = forward64(t["X"], t["weight"], t["residual"], dtype)
    r = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS)
    assert torch.equal(r.H.double(), h) and (r.H is t["X"] or residual or r.H.data_ptr() == t["X"].data_ptr())
    near = (terms(d) / 2 + 6) * STEP
    assert ((r.rstd.double() / rstd[:, 0] - 1).abs() <= near).all()
    assert r.Y.dtype == dtype and ((r.Y.double() - y).abs() <= y.abs() * (near + 2 * STEP + eight.HALF[dtype] * 1.01)).all()
    assert r.Y8 is None and r.scales is None


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("f8", eight.F8)
@pytest.mark.parametrize("n,d", SHAPES)
def test_rows_in_8_bits(n, d, f8, scale_dtype):
    """Scales and data follow from the unrounded Y: a scale is a few steps of fp32 off at most (a power of two: the one of a maximum
    that near), a value half a step of its format."""
    for dtype in DTYPES:
        t = inputs(n, d, dtype, seed=1)
        h, rstd, y = forward64(t["X"], t["weight"], t["residual"], dtype)
        r = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS, f8=f8, scale_dtype=scale_dtype)
        near = (terms(d) / 2 + 8) * STEP
        y, s = y.cpu(), eight.scale64(r.scales)
        wide = torch.nn.functional.pad(y, (0, eight.blocks(d) * 128 - d)).view(n, -1, 128)
        amax = wide.abs().amax(2).t()
        if scale_dtype == torch.float32:
            want = (amax / eight.TOP[f8]).clamp(min=2.0 ** -126)
            assert ((s / want - 1).abs() <= near + STEP).all()
        else:
            low, high = (eight.scale_of((amax * f).float(), f8, scale_dtype).double() for f in (1 - near - STEP, 1 + near + STEP))
            assert ((s >= low) & (s <= high)).all()
        v = eight.values_rows(r.Y8, r.scales)
        unit = s.t().repeat_interleave(128, 1)[:, :d]
        assert ((v - y).abs() <= y.abs() * (eight.HALF[f8] * 1.001 + near) + unit * eight.LEAST[f8] / 2).all()
        plain = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS)
        assert torch.equal(plain.Y, r.Y) and torch.equal(plain.H, r.H) and torch.equal(plain.rstd, r.rstd)
        only = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS, need_Y=False, f8=f8, scale_dtype=scale_dtype)
        assert only.Y is None and torch.equal(eight.bytes_of(only.Y8), eight.bytes_of(r.Y8))


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("f8", eight.F8)
@pytest.mark.parametrize("n,d,residual", [(700, 1001, False), (500, 768, True), (300, 2500, True), (90, 6001, False), (20, 40000, True)])
def test_8_bit_rows_are_those_of_the_result_in_64_bits(n, d, residual, f8, scale_dtype):
    """Every scale and byte: Y is made to about 2^-46, and of some 2^20 quotients none lies that near to a number half way between two."""
    for dtype in DTYPES:
        t = inputs(n, d, dtype, residual, seed=5)
        _, _, y = forward64(t["X"], t["weight"], t["residual"], dtype)
        r = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS, need_Y=False, f8=f8, scale_dtype=scale_dtype)
        y = torch.nn.functional.pad(y.cpu(), (0, eight.blocks(d) * 128 - d)).view(n, -1, 128)
        s = (y.abs().amax(2) / eight.TOP[f8]).clamp(min=2.0 ** -126).float()
        if scale_dtype == torch.float8_e8m0fnu:
            m, e = torch.frexp(s)
            s = torch.ldexp(torch.ones_like(s), torch.where(m == 0.5, e - 1, e))
        assert torch.equal(eight.scale64(r.scales), s.t().double())
        want = (y / s[..., None].double()).float().to(f8).view(n, -1)[:, :d]
        assert torch.equal(eight.bytes_of(r.Y8), eight.bytes_of(want))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", SHAPES + [(600, 768), (2100, 256), (1030, 4096), (513, 1001)])
def test_backward(n, d, dtype):
    for with_dh in (False, True):
        t = inputs(n, d, dtype, seed=2)
        r = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS)
        dX, dw = rmm.rmm_rms_norm_backward(t["dY"], r.H, t["weight"], r.rstd, t["dH"] if with_dh else None)
        h, rstd, _ = forward64(t["X"], t["weight"], t["residual"], dtype)
        dy, hat = t["dY"].double(), h * rstd
        g = dy * t["weight"].double()
        mean, size = (g * hat).mean(1, keepdim=True), (g * hat).abs().mean(1, keepdim=True)
        want = rstd * (g - hat * mean) + (t["dH"].double() if with_dh else 0)
        # rstd is off by `near`, and with it hat twice in the product; the sum over the row adds its terms
        near = (terms(d) / 2 + 8) * STEP
        off = rstd * (4 * near * (g.abs() + hat.abs() * size) + terms(d) * STEP * hat.abs() * size) + 2 * STEP * want.abs()
        assert dX.dtype == dtype and ((dX.double() - want).abs() <= off + eight.HALF[dtype] * 1.01 * want.abs()).all()
        dw64, dw_size = (dy * hat).sum(0), (dy * hat).abs().sum(0)
        assert dw.dtype == dtype
        assert ((dw.double() - dw64).abs() <= dw_size * (n / 16 + 80 + near / STEP) * STEP + eight.HALF[dtype] * 1.01 * dw64.abs()).all()
        again = rmm.rmm_rms_norm_backward(t["dY"], r.H, t["weight"], r.rstd, t["dH"] if with_dh else None)
        assert torch.equal(again[0], dX) and torch.equal(again[1], dw)
        alone = rmm.rmm_rms_norm_backward(t["dY"], r.H, t["weight"], r.rstd, t["dH"] if with_dh else None, need_dweight=False)
        assert alone[1] is None and torch.equal(alone[0], dX)
        alone = rmm.rmm_rms_norm_backward(t["dY"], r.H, t["weight"], r.rstd, need_dX=False)
        assert alone[0] is None and torch.equal(alone[1], dw)


def test_gradient_against_differences():
    n, d, step = 3, 40, 1e-5
    t = {k: v.cpu().double() for k, v in inputs(n, d, torch.float32, seed=3).items()}

    def loss(X, w):
        return ((X * (1 / torch.sqrt((X * X).mean(1, keepdim=True) + EPS)) * w) * t["dY"]).sum()

    dev = {k: v.float().to(DEV) for k, v in t.items()}
    r = rmm.rmm_rms_norm(dev["X"], dev["weight"], None, EPS)
    dX, dw = rmm.rmm_rms_norm_backward(dev["dY"], r.H, dev["weight"], r.rstd)
    for i, j in ((0, 0), (1, 17), (2, 39)):
        e = torch.zeros(n, d, dtype=torch.float64)
        e[i, j] = step
        slope = (loss(t["X"] + e, t["weight"]) - loss(t["X"] - e, t["weight"])) / (2 * step)
        assert abs(float(dX[i, j]) - float(slope)) < 1e-4 * max(1.0, abs(float(slope)))
        slope = (loss(t["X"], t["weight"] + e[i]) - loss(t["X"], t["weight"] - e[i])) / (2 * step)
        assert abs(float(dw[j]) - float(slope)) < 1e-4 * max(1.0, abs(float(slope)))


@pytest.mark.parametrize("d", [64, 3000, 40000])
def test_rows_of_zeros_infinities_and_nan_stay_by_themselves(d):
    X = torch.randn(6, d, device=DEV)
    X[1] = 0
    X[2, d // 2] = float("inf")
    X[3, 0] = float("nan")
    w = torch.ones(d, device=DEV)
    r = rmm.rmm_rms_norm(X, w, None, EPS, f8=torch.float8_e4m3fn)
    h, _, y = forward64(X, w, None, torch.float32)
    good = [0, 4, 5]
    assert ((r.Y[good].double() - y[good]).abs() <= 1e-5 * y[good].abs()).all()
    assert (r.Y[1] == 0).all() and (r.Y8[1].float() == 0).all() and abs(float(r.rstd[1]) - EPS ** -0.5) < 1e-3
    assert torch.equal(r.Y[2].isnan(), y[2].isnan()) and r.Y[3].isnan().all()
    assert torch.isfinite(r.scales[:, good]).all() and not torch.isfinite(r.scales[:, 3]).any()
    dY = torch.randn(6, d, device=DEV)
    dX, _ = rmm.rmm_rms_norm_backward(dY, X, w, r.rstd, need_dweight=False)
    assert torch.isfinite(dX[[0, 1, 4, 5]]).all() and dX[3].isnan().all()


def test_large_and_small_values():
    """Squares must not overflow where the mean is a number; eps decides for rows far below its root."""
    d = 256
    X = torch.randn(3, d, device=DEV)
    X[0] *= 1e17
    X[1] *= 1e-12
    w = torch.ones(d, device=DEV)
    r = rmm.rmm_rms_norm(X, w, None, EPS)
    _, _, y = forward64(X, w, None, torch.float32)
    assert ((r.Y.double() - y).abs() <= 1e-5 * y.abs() + 1e-30).all()


@pytest.mark.parametrize("d", [768, 6000, 40000])
def test_update_in_place(d):
    """H may be the buffer of the residual, dX that of dY."""
    from paper_2201_13195_amd import binding
    t = inputs(50, d, torch.bfloat16, seed=5)
    want = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS)
    res, Y = t["residual"].clone(), torch.empty_like(t["X"])
    L, s = rmm.load_library(), binding._stream(res)
    assert L.rmm_rms_norm(50, d, 1, EPS, t["X"].data_ptr(), res.data_ptr(), t["weight"].data_ptr(), res.data_ptr(), Y.data_ptr(), None, None, s) == 0
    assert torch.equal(res, want.H) and torch.equal(Y, want.Y)
    dX, dw = rmm.rmm_rms_norm_backward(t["dY"], want.H, t["weight"], want.rstd, t["dH"])
    dY, out = t["dY"].clone(), torch.empty_like(dw)
    ws = torch.empty(L.rmm_rms_norm_workspace_bytes(50, d, 1), dtype=torch.uint8, device=DEV)
    assert L.rmm_rms_norm_backward(50, d, 1, dY.data_ptr(), t["dH"].data_ptr(), want.H.data_ptr(), t["weight"].data_ptr(), want.rstd.data_ptr(),
                                   dY.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(), s) == 0
    assert torch.equal(dY, dX) and torch.equal(out, dw)


def test_without_h_the_residual_is_still_added():
    from paper_2201_13195_amd import binding
    for d in (300, 40000):
        t = inputs(5, d, torch.bfloat16, seed=6)
        want = rmm.rmm_rms_norm(t["X"], t["weight"], t["residual"], EPS)
        Y = torch.empty_like(t["X"])
        assert rmm.load_library().rmm_rms_norm(5, d, 1, EPS, t["X"].data_ptr(), t["residual"].data_ptr(), t["weight"].data_ptr(), None,
                                               Y.data_ptr(), None, None, binding._stream(Y)) == 0
        assert torch.equal(Y, want.Y)


def test_long_matrix_passes_32_bit_offsets():
    n, d = (1 << 31) // 2048 + 5, 2048
    X = torch.ones(n, d, dtype=torch.bfloat16, device=DEV)
    X[-1] = torch.linspace(-3, 3, d, device=DEV)
    w = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    r = rmm.rmm_rms_norm(X, w, None, EPS, f8=torch.float8_e4m3fn)
    few = rmm.rmm_rms_norm(X[-3:].contiguous(), w, None, EPS, f8=torch.float8_e4m3fn)
    assert torch.equal(r.Y[-3:], few.Y) and torch.equal(eight.bytes_of(r.Y8[-3:]), eight.bytes_of(few.Y8)) and torch.equal(r.scales[:, -3:], few.scales)
    dX, dw = rmm.rmm_rms_norm_backward(r.Y, X, w, r.rstd)
    dX3, _ = rmm.rmm_rms_norm_backward(few.Y, X[-3:].contiguous(), w, few.rstd)
    assert torch.equal(dX[-3:], dX3)


@pytest.mark.parametrize("f8", eight.F8)
def test_powers_of_two_at_the_border_between_two(f8):
    """The largest magnitude of each block lies 0.55 to 0.85 steps of fp32 above the format's largest number: rounded by itself it is one
    step above it and asks for the next power, but its quotient, rounded to fp32, is still 1 (up to 0.875 steps: half a step of 1)."""
    d, top = 64 * 128, eight.TOP[f8]
    X = torch.randn(1, d, generator=torch.Generator().manual_seed(11))
    hat = X.double() / torch.sqrt((X.double() ** 2).mean() + EPS)
    step = top * 2.0 ** -23 / 1.75                        # of fp32, at top = 1.75 * 2^k
    weight = torch.ones(d)
    for b in range(d // 128):
        part = hat[0, b * 128:(b + 1) * 128].abs()
        w = ((top + 0.7 * step) / part).float()
        above = (part * w.double() - top) / step
        fits = ((above > 0.55) & (above < 0.85) & (part > 0.1)).nonzero()
        assert len(fits)
        weight[b * 128 + int(fits[0])] = w[int(fits[0])]
    y = (hat * weight.double()).view(-1, 128)
    assert (y.abs().amax(1) > top).all() and (y.abs().amax(1).float() > top).all()
    r = rmm.rmm_rms_norm(X.to(DEV), weight.to(DEV), None, EPS, need_Y=False, f8=f8, scale_dtype=torch.float8_e8m0fnu)
    assert torch.equal((y.abs().amax(1) / top).float(), torch.ones(d // 128))
    assert (eight.scale64(r.scales) == 1).all()
    assert torch.equal(eight.bytes_of(r.Y8), eight.bytes_of(y.float().to(f8).view(1, d)))


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("size,eps", [(1e25, EPS), (1e29, EPS), (1e-25, 0.0), (1e-29, 0.0)])
def test_8_bit_rows_of_very_large_and_very_small_rows(size, eps, scale_dtype):
    """Rows whose mean square is no number of fp32: scales and bytes are those of the result in 64 bits all the same."""
    n, d, f8 = 60, 700, torch.float8_e4m3fn
    X = torch.randn(n, d, generator=torch.Generator().manual_seed(12)) * size
    w = 1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(13))
    r = rmm.rmm_rms_norm(X.to(DEV), w.to(DEV), None, eps, need_Y=False, f8=f8, scale_dtype=scale_dtype)
    y = X.double() / torch.sqrt((X.double() ** 2).mean(1, keepdim=True) + eps) * w.double()
    y = torch.nn.functional.pad(y, (0, eight.blocks(d) * 128 - d)).view(n, -1, 128)
    s = (y.abs().amax(2) / eight.TOP[f8]).float()
    if scale_dtype == torch.float8_e8m0fnu:
        m, e = torch.frexp(s)
        s = torch.ldexp(torch.ones_like(s), torch.where(m == 0.5, e - 1, e))
    assert torch.equal(eight.scale64(r.scales), s.t().double())
    want = (y / s[..., None].double()).float().to(f8).view(n, -1)[:, :d]
    assert torch.equal(eight.bytes_of(r.Y8), eight.bytes_of(want))


@pytest.mark.parametrize("n,d,dtype", [((1 << 31) // 2048 + 5, 2048, torch.bfloat16), (300001, 257, torch.float32), (60000, 5000, torch.bfloat16),
                                       (6001, 20000, torch.float32), (30000, 16392, torch.bfloat16)])
def test_weight_gradient_of_many_rows(n, d, dtype):
    """A thread adds at most n / 64 rows (long rows; n / 256 others), and up to 512 such sums follow.  The roundings are independent, each at
    most 2^-24 of a partial sum, which in the mean is no more than the root of the sum of squares; eight more for what is summed."""
    g = torch.Generator(DEV).manual_seed(n)
    X = torch.empty(n, d, dtype=dtype, device=DEV)
    dY = torch.empty(n, d, dtype=dtype, device=DEV)
    for t in (X, dY):
        t.normal_(generator=g)
    w = torch.ones(d, dtype=dtype, device=DEV)
    rstd = rmm.rmm_rms_norm(X, w, None, EPS).rstd
    _, dw = rmm.rmm_rms_norm_backward(dY, X, w, rstd, need_dX=False)
    want, squares = torch.zeros(d, dtype=torch.float64, device=DEV), torch.zeros(d, dtype=torch.float64, device=DEV)
    for at in range(0, n, 1 << 14):
        h, dy = X[at:at + (1 << 14)].double(), dY[at:at + (1 << 14)].double()
        part = dy * h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        want += part.sum(0)
        squares += part.square().sum(0)
    adds = n / (64 if d > 16384 else 256) + 512
    off = float((dw.double() - want).norm())
    assert off <= (adds ** 0.5 + 8) * STEP * float(squares.sum().sqrt()) + 1.01 * eight.HALF[dtype] * float(want.norm())
