"""GPU: Y = X W^T (+ bias) of 8-bit operands against the product of their values in 64 bits."""
import pytest
import torch

import eight
import paper_2201_13195_amd as rmm
from test_linear8_plan import KERNELS

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2


def operands(n, d_in, d_out, f8=E4, scale_dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(seed + n + 31 * d_in + 77 * d_out)
    X = torch.randn(n, d_in, generator=g) * torch.exp(torch.randn(n, 1, generator=g))
    W = torch.randn(d_out, d_in, generator=g) / d_in ** 0.5
    x = rmm.rmm_quantize8(X.bfloat16().to(DEV), f8=f8, scale_dtype=scale_dtype)
    w = rmm.rmm_quantize8_weight(W.bfloat16().to(DEV), scale_dtype=scale_dtype)
    return x, w, torch.randn(d_out, generator=g)


def check(x, w, bias, dtype, Y):
    """Every element within what the roundings allow: d_in products are summed in fp32 in some order (each sum and each product
    with a scale is at most a step off, 2^-23 of the sum of magnitudes; three more for the scales and the bias), then rounded once
    to the output.  A bf16 output's sums come from the 8-bit matrix instructions, which cut up to seven of eight products to 2^-13 of
    the largest one: 7 * 2^-13 of the sum of magnitudes at most, and over many elements, whose cuts are independent, 2^-13 of the
    norm of what is summed."""
    X, W = eight.values_rows(*x).to(DEV), eight.values_weight(*w).to(DEV)
    b = torch.zeros(W.shape[0], dtype=torch.float64, device=DEV) if bias is None else bias.double().to(DEV)
    want, size = X @ W.t() + b, X.abs() @ W.abs().t() + b.abs()
    off = (Y.double() - want).abs()
    assert Y.dtype == dtype and torch.isfinite(Y).all()
    bound = (X.shape[1] + 4) * 2.0 ** -23 * size + eight.HALF[dtype] * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -140
    if dtype == torch.bfloat16:
        bound += 7 * 2.0 ** -13 * size
        assert float(off.norm()) <= (eight.HALF[dtype] + 2.0 ** -13) * float(want.norm()) + 2.0 ** -13 * float((X.square() @ W.square().t()).sum().sqrt())
    assert (off <= bound).all(), float((off / bound).max())


SHAPES = [(1, 1, 1), (1, 128, 16), (1, 1000, 1111), (2, 129, 17), (7, 4096, 100), (16, 512, 512), (17, 640, 33), (24, 4096, 1024),
          (33, 127, 257), (64, 1024, 64), (65, 100, 300), (100, 2053, 129), (130, 384, 130), (257, 768, 768), (300, 16, 1300),
          (515, 1029, 261), (1024, 256, 640), (1277, 344, 344)]


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in,d_out", SHAPES)
def test_shapes(n, d_in, d_out, scale_dtype):
    for f8, dtype, with_bias in ((E4, torch.bfloat16, True), (E5, torch.float32, False), (E4, torch.float32, True), (E5, torch.bfloat16, True)):
        x, w, bias = operands(n, d_in, d_out, f8, scale_dtype)
        bias = bias.to(dtype).to(DEV) if with_bias else None
        check(x, w, bias, dtype, rmm.rmm_linear8(*x, *w, bias=bias, dtype=dtype))


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("shape", [shape for shape, _, _ in KERNELS])
def test_every_kernel(shape, scale_dtype):
    for f8, dtype, with_bias in ((E4, torch.bfloat16, False), (E5, torch.bfloat16, True), (E4, torch.float32, True), (E5, torch.float32, False)):
        x, w, bias = operands(*shape, f8, scale_dtype)
        bias = bias.to(dtype).to(DEV) if with_bias else None
        check(x, w, bias, dtype, rmm.rmm_linear8(*x, *w, bias=bias, dtype=dtype))


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in,d_out", [(4096, 1024, 1536), (2049, 520, 4100), (8192, 264, 2048), (3000, 4096, 1025)])
def test_large(n, d_in, d_out, scale_dtype):
    x, w, bias = operands(n, d_in, d_out, E4, scale_dtype)
    check(x, w, None, torch.bfloat16, rmm.rmm_linear8(*x, *w))
    check(x, w, bias.to(DEV), torch.float32, rmm.rmm_linear8(*x, *w, bias=bias.to(DEV), dtype=torch.float32))


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n", [1, 20, 150, 700, 2500])
def test_small_whole_numbers_are_exact(n, scale_dtype):
    """Data of -2 .. 2 and scales of powers of two: every sum is a number of fp32, so the result is exact in any order."""
    g = torch.Generator().manual_seed(n)
    d_in, d_out = 1000, 770
    X, W = torch.randint(-2, 3, (n, d_in), generator=g).float(), torch.randint(-2, 3, (d_out, d_in), generator=g).float()
    xs = torch.exp2(torch.randint(-3, 4, (eight.blocks(d_in), (n + 15) // 16 * 16), generator=g).float())
    ws = torch.exp2(torch.randint(-3, 4, (eight.blocks(d_out), eight.blocks(d_in)), generator=g).float())
    pitched = torch.zeros(n, 1008).to(E4)
    pitched.view(torch.uint8)[:, :d_in] = X.to(E4).view(torch.uint8)
    wide = torch.zeros(d_out, 1008).to(E4)
    wide.view(torch.uint8)[:, :d_in] = W.to(E4).view(torch.uint8)
    x = pitched.to(DEV)[:, :d_in], xs.to(scale_dtype).to(DEV)[:, :n]
    w = wide.to(DEV)[:, :d_in], ws.to(scale_dtype).to(DEV)
    want = eight.values_rows(*x) @ eight.values_weight(*w).t()
    assert torch.equal(rmm.rmm_linear8(*x, *w, dtype=torch.float32).cpu().double(), want)


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in", [(3, 1000), (40, 1001), (300, 1015), (2100, 999), (2100, 65)])
def test_what_lies_behind_the_rows_is_not_read_as_numbers(n, d_in, scale_dtype):
    """NaN bytes behind the columns of both operands and NaN scales behind the rows change nothing."""
    x, w, _ = operands(n, d_in, 520, E4, scale_dtype)
    want = rmm.rmm_linear8(*x, *w)
    wide = []
    for t in (x[0], w[0]):
        b = torch.full((t.shape[0] + 1, 1152), 0x7F, dtype=torch.uint8, device=DEV)
        b[:t.shape[0], :d_in] = t.view(torch.uint8)
        wide.append(b.view(E4)[:t.shape[0], :d_in])
    xs = torch.full((x[1].shape[0], x[1].stride(0) + 64), float("nan"), device=DEV).to(scale_dtype)
    raw = torch.float32 if scale_dtype == torch.float32 else torch.uint8
    xs.view(raw)[:, :n] = x[1].view(raw)
    assert torch.equal(rmm.rmm_linear8(wide[0], xs[:, :n], wide[1], w[1]), want)


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n", [1, 30, 500, 2300])
def test_blocks_that_are_no_numbers_stay_in_their_row(n, scale_dtype):
    """An infinity or NaN in one token, one weight: NaN in that row and that column's block, numbers elsewhere."""
    g = torch.Generator().manual_seed(3)
    X, W = torch.randn(n, 384, generator=g), torch.randn(300, 384, generator=g)
    X[n // 2, 200] = float("inf")
    W[150, 3] = float("nan")
    x = rmm.rmm_quantize8(X.to(DEV), scale_dtype=scale_dtype)
    w = rmm.rmm_quantize8_weight(W.to(DEV), scale_dtype=scale_dtype)
    Y = rmm.rmm_linear8(*x, *w, dtype=torch.float32).cpu()
    bad = Y.isnan()
    want = torch.zeros(n, 300, dtype=torch.bool)
    want[n // 2] = True
    want[:, 128:256] = True
    assert torch.equal(bad, want) and torch.isfinite(Y[~want]).all()


def test_the_gradient_is_the_product_with_the_transposed_weights():
    n, d_in, d_out = 333, 520, 392
    g = torch.Generator().manual_seed(9)
    W, dY = torch.randn(d_out, d_in, generator=g).to(DEV), torch.randn(n, d_out, generator=g).to(DEV)
    for scale_dtype in eight.SCALES:
        w = rmm.rmm_quantize8_weight(W, scale_dtype=scale_dtype, transposed=True)
        dy = rmm.rmm_quantize8(dY, f8=E5, scale_dtype=scale_dtype)
        dX = rmm.rmm_linear8(*dy, *w[2:], dtype=torch.float32)
        check(dy, w[2:], None, torch.float32, dX)
        want = eight.values_rows(*dy) @ eight.values_weight(*w[:2])
        assert float((dX.cpu().double() - want).norm() / want.norm()) < 1e-5


def test_same_bits_every_time_and_into_a_given_buffer():
    for n, d_in, d_out in ((1, 4096, 1024), (24, 4096, 1024), (333, 1000, 1111), (2500, 1024, 1024)):
        x, w, _ = operands(n, d_in, d_out)
        Y = rmm.rmm_linear8(*x, *w)
        out = torch.full((n, d_out), float("nan"), dtype=torch.bfloat16, device=DEV)
        assert rmm.rmm_linear8(*x, *w, Y=out).data_ptr() == out.data_ptr()
        assert torch.equal(out, Y) and torch.equal(rmm.rmm_linear8(*x, *w), Y)


def test_rows_of_a_larger_batch_are_the_same_matrix():
    """Views of rows and of scales (what a batch cut in two holds) are operands as they are."""
    x, w, _ = operands(96, 512, 256)
    Y = rmm.rmm_linear8(*x, *w, dtype=torch.float32)
    part = rmm.rmm_linear8(x[0][16:80], x[1][:, 16:80], *w, dtype=torch.float32)
    check((x[0][16:80], x[1][:, 16:80]), w, None, torch.float32, part)
    assert torch.allclose(part, Y[16:80], rtol=1e-5, atol=1e-5)


def test_on_another_stream():
    x, w, _ = operands(300, 512, 512)
    want = rmm.rmm_linear8(*x, *w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = rmm.rmm_linear8(*x, *w)
    s.synchronize()
    assert torch.equal(got, want)


def test_large_offsets():
    """Operands and output beyond 2^31 elements."""
    n, d_in, d_out = 140000, 16400, 16
    x8 = torch.zeros(n, d_in, dtype=torch.uint8, device=DEV)
    x8[-1] = torch.randint(0, 0x70, (d_in,), dtype=torch.uint8, device=DEV)
    xs = torch.ones(eight.blocks(d_in), n, device=DEV)
    w = rmm.rmm_quantize8_weight(torch.randn(d_out, d_in, device=DEV))
    Y = rmm.rmm_linear8(x8.view(E4), xs, *w, dtype=torch.float32)
    check((x8.view(E4)[-1:], xs[:, -1:]), w, None, torch.float32, Y[-1:])
    assert (Y[:-1] == 0).all()
    del x8, Y
    n, d_in, d_out = 70000, 16, 33000
    x, w, _ = operands(n, d_in, 128)
    w8, ws = w[0].view(torch.uint8).repeat(258, 1)[:d_out], w[1].repeat(258, 1)
    Y = rmm.rmm_linear8(*x, w8.view(E4), ws)
    first = rmm.rmm_linear8(*x, *w)
    assert torch.equal(Y[-300:, :128], first[-300:]) and torch.equal(Y[-300:, 128 * 200:128 * 201], first[-300:])


# kernels: 64x32, 64 x 128 tiles twice, 128 split, 128, 256; then those of few tokens
TILES = [(300, 1000, 3001), (2100, 999, 520), (300, 1000, 3501), (3000, 2501, 1000), (2100, 300, 1500), (4300, 1001, 4090),
         (5, 1001, 3000), (40, 2001, 1001), (128, 1111, 4000), (16, 1001, 9000), (30, 2001, 9000), (60, 1001, 9000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in,d_out", TILES)
def test_tiles_take_nothing_from_behind_their_operands(n, d_in, d_out, scale_dtype, dtype):
    """NaN behind columns, rows and scales of both operands, and around a Y that is given: the same bits, and nothing else written."""
    x, w, _ = operands(n, d_in, d_out, E4, scale_dtype)
    want = rmm.rmm_linear8(*x, *w, dtype=dtype)
    raw = torch.float32 if scale_dtype == torch.float32 else torch.uint8
    data, scales = [], []
    for t, s, high, wide in ((x[0], x[1], 0, 80), (w[0], w[1], 1, 3)):
        b = torch.full((t.shape[0] + 256, (d_in + 15) // 16 * 16 + 160), 0x7F, dtype=torch.uint8, device=DEV)
        b[:t.shape[0], :d_in] = t.view(torch.uint8)
        data.append(b.view(E4)[:t.shape[0], :d_in])
        pitch = (s.shape[1] + wide + 15) // 16 * 16
        c = torch.full((s.shape[0] + high + 1, pitch), float("nan"), device=DEV).to(scale_dtype)
        c.view(raw)[:s.shape[0], :s.shape[1]] = s.view(raw)
        scales.append(c[:s.shape[0], :s.shape[1]])
    around = torch.full(((n + 300) * d_out,), 7.0, dtype=dtype, device=DEV)
    Y = around[:n * d_out].view(n, d_out)
    rmm.rmm_linear8(data[0], scales[0], data[1], scales[1], dtype=dtype, Y=Y)
    assert torch.equal(Y, want) and bool((around[n * d_out:] == 7.0).all())
    assert torch.equal(rmm.rmm_linear8(*x, *w, dtype=dtype), want)


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in,d_out", TILES)
def test_no_numbers_in_one_block_of_a_tile(n, d_in, d_out, scale_dtype):
    """A token with an infinity in each block in turn, and no others, is NaN."""
    x, w, _ = operands(n, d_in, d_out, E4, scale_dtype)
    want = rmm.rmm_linear8(*x, *w)
    blocks = (d_in + 127) // 128
    tokens = torch.arange(blocks) * (n // blocks)
    X = torch.zeros(n, d_in)
    X[tokens, torch.arange(blocks) * 128 + 5] = float("inf")
    bad = rmm.rmm_quantize8(X.to(DEV), scale_dtype=scale_dtype)
    data, scales = x[0].clone(), x[1].clone()
    raw = torch.float32 if scale_dtype == torch.float32 else torch.uint8
    for b, t in enumerate(tokens.tolist()):
        data.view(torch.uint8)[t, 128 * b:128 * b + 128] = bad[0].view(torch.uint8)[t, 128 * b:128 * b + 128]
        scales.view(raw)[b, t] = bad[1].view(raw)[b, t]
    wide = rmm.rmm_quantize8(torch.zeros(n, d_in, device=DEV), scale_dtype=scale_dtype)
    wide[0].view(torch.uint8).copy_(data.view(torch.uint8))
    wide[1].view(raw).copy_(scales.view(raw))
    Y = rmm.rmm_linear8(*wide, *w)
    assert bool(Y[tokens.to(DEV)].isnan().all())
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[tokens.to(DEV)] = False
    assert torch.equal(Y[others], want[others])


def test_every_tile_kernel_in_a_graph_replayed():
    """All in one capture, on inputs that change between the replays; two of them side by side on streams of their own."""
    ops = [operands(*shape, E4, eight.SCALES[i % 2]) for i, shape in enumerate(TILES)]
    out = [torch.empty(x[0].shape[0], w[0].shape[0], dtype=torch.bfloat16, device=DEV) for x, w, _ in ops]

    def run():
        for (x, w, _), y in zip(ops, out):
            rmm.rmm_linear8(*x, *w, Y=y)

    side, beside = torch.cuda.Stream(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for step in range(3):
        for x, _, _ in ops:
            raw = x[0].view(torch.uint8)
            raw.copy_(raw.roll(1 + step, 0))
        want = [rmm.rmm_linear8(*x, *w) for x, w, _ in ops]
        for y in out:
            y.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        beside.wait_stream(torch.cuda.current_stream())
        again = [torch.empty_like(y) for y in out]
        with torch.cuda.stream(beside):
            for (x, w, _), y in zip(ops, again):
                rmm.rmm_linear8(*x, *w, Y=y)
        run_here = [rmm.rmm_linear8(*x, *w) for x, w, _ in ops]
        torch.cuda.synchronize()
        for a, b, c, d in zip(want, out, again, run_here):
            assert torch.equal(a, b) and torch.equal(a, c) and torch.equal(a, d)


def test_more_tiles_than_a_launch_has_work_groups():
    """2^30 tokens of one block: the work-groups go on from tile to tile."""
    n, d_in, d_out = (1 << 30) + 37, 16, 3
    data = torch.randint(0, 0x60, (1 << 20, 16), dtype=torch.uint8, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    X = torch.empty((n, 16), dtype=torch.uint8, device=DEV)
    for at in range(0, n, 1 << 20):
        here = min(1 << 20, n - at)
        X[at:at + here] = data[:here] ^ ((at >> 20) & 3)
    xs = torch.full((1, (n + 15) // 16 * 16), 127, dtype=torch.uint8, device=DEV)[:, :n]
    xs[0, 5::7] = 126
    w = rmm.rmm_quantize8_weight(torch.randn(d_out, d_in, device=DEV), scale_dtype=torch.float8_e8m0fnu)
    Y = rmm.rmm_linear8(X.view(E4), xs.view(torch.float8_e8m0fnu), *w)
    for at in (0, (1 << 22) * 32 - 160, (1 << 27) + 64, (1 << 29) + 48, (1 << 30) - 2000):
        part = slice(at, min(at + 2048, n))
        want = rmm.rmm_linear8(X[part].view(E4), xs[:, part].view(torch.float8_e8m0fnu), *w)
        assert torch.equal(Y[part], want)


def powers(n, d_in, d_out, X, W, f8, ex, ew):
    """Operands with these data and powers of two: 2^(ex - 3 (b mod 4)) for X's block b, 2^(ew + 3 (b mod 4)) for W's."""
    by = 3 * (torch.arange(eight.blocks(d_in)) % 4)

    def pitched(A, f8):
        a = torch.zeros(A.shape[0], (d_in + 15) // 16 * 16, dtype=torch.uint8)
        a[:, :d_in] = A.to(f8).view(torch.uint8)
        return a.to(DEV).view(f8)[:, :d_in]
    xs = (127 + ex - by).to(torch.uint8)[:, None].expand(-1, (n + 15) // 16 * 16).contiguous()
    ws = (127 + ew + by).to(torch.uint8)[None].expand(eight.blocks(d_out), -1).contiguous()
    e8m0 = torch.float8_e8m0fnu
    return (pitched(X, f8), xs.to(DEV).view(e8m0)[:, :n]), (pitched(W, E4), ws.to(DEV).view(e8m0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d_in,d_out", [shape for shape, _, _ in KERNELS])
def test_scales_whose_product_is_no_number_of_fp32(n, d_in, d_out, dtype):
    """Powers of two of both sides that multiply to more than fp32's largest number, or less than its smallest, where the result is one of
    fp32's: with whole numbers it is exact, as no sum of up to 4 d_in of them needs more than 24 bits."""
    g = torch.Generator().manual_seed(n + d_in)
    for f8 in (E4, E5):
        X, W = torch.randint(-2, 3, (n, d_in), generator=g).float(), torch.randint(-2, 3, (d_out, d_in), generator=g).float()
        # 2^-18 of whole numbers up to 4 d_in <= 2^15, times 2^130
        x, w = powers(n, d_in, d_out, X * 2.0 ** -9, W * 2.0 ** -9, f8, 100, 30)
        want = eight.values_rows(*x) @ eight.values_weight(*w).t()
        assert torch.equal(rmm.rmm_linear8(*x, *w, dtype=dtype).cpu(), want.to(dtype))
        # zeros stay zeros, whatever the scales
        x, w = powers(n, d_in, d_out, torch.zeros(n, d_in), W, f8, 120, 110)
        assert (rmm.rmm_linear8(*x, *w, dtype=dtype) == 0).all()
        # 384^2 and more for each product, times 2^-150: a block's sum of 128 is one of fp32's normal numbers
        X, W = 448 - 32 * torch.randint(0, 2, (n, d_in), generator=g).float(), 448 - 32 * torch.randint(0, 3, (d_out, d_in), generator=g).float()
        x, w = powers(n, d_in, d_out, X, W, f8, -90, -60)
        X64, W64 = eight.values_rows(*x), eight.values_weight(*w)
        Y = rmm.rmm_linear8(*x, *w, dtype=dtype).cpu().double()
        want = X64 @ W64.t()
        # (the sum as in `check`; a last block of fewer may be less than 2^-126, and lost)
        bound = (d_in + 4) * 2.0 ** -23 * want + eight.HALF[dtype] * want * (1 + 2.0 ** -8) + 2.0 ** -126
        if dtype == torch.bfloat16:
            bound += 7 * 2.0 ** -13 * want
        assert ((Y - want).abs() <= bound).all(), float(((Y - want).abs() / bound).max())


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in,d_out", [shape for shape, _, _ in KERNELS])
def test_fp32_results_hold_what_stands_beside_a_large_product(n, d_in, d_out, scale_dtype):
    """One product of 2^15 in each eight contraction elements, the others 1, -1 or 0: the 8-bit matrix instruction would cut those off.
    No sum needs more than 24 bits, so the result is exact."""
    g = torch.Generator().manual_seed(n + d_out)
    for f8 in (E4, E5):
        X, W = torch.randint(-1, 2, (n, d_in), generator=g).float(), torch.randint(-1, 2, (d_out, d_in), generator=g).float()
        at = torch.arange(0, d_in - 7, 8) + torch.randint(0, 8, (d_in // 8,), generator=g)
        X[:, at], W[:, at] = X[:, at] * 256, W[:, at] * 128
        x, w = powers(n, d_in, d_out, X, W, f8, 3, -3)
        if scale_dtype == torch.float32:
            xs = torch.zeros(x[1].shape[0], x[1].stride(0), device=DEV)
            xs[:, :n] = x[1].float()
            x, w = (x[0], xs[:, :n]), (w[0], w[1].float())
        want = eight.values_rows(*x) @ eight.values_weight(*w).t()
        assert torch.equal(rmm.rmm_linear8(*x, *w, dtype=torch.float32).cpu().double(), want)


@pytest.mark.parametrize("scale_dtype", eight.SCALES)
@pytest.mark.parametrize("n,d_in,d_out", [shape for shape, _, _ in KERNELS])
def test_fp32_results_in_the_mean(n, d_in, d_out, scale_dtype):
    """The roundings of d_in sums, and of four more for scales and product, are independent: each at most 2^-23 of a partial sum, which for
    products of both signs is no more than the root of the sum of their squares in the mean."""
    for f8 in (E4, E5):
        x, w, _ = operands(n, d_in, d_out, f8, scale_dtype)
        X, W = eight.values_rows(*x).to(DEV), eight.values_weight(*w).to(DEV)
        off = rmm.rmm_linear8(*x, *w, dtype=torch.float32).double() - X @ W.t()
        assert float(off.norm()) <= (d_in + 4) ** 0.5 * 2.0 ** -23 * float((X.square() @ W.square().t()).sum().sqrt())
