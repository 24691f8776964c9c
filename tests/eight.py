"""Plain forms of the 8-bit operators on the CPU, for the tests: quantisation from its definition, values in 64 bits."""
import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
F8 = [torch.float8_e4m3fn, torch.float8_e5m2]
SCALES = [torch.float32, torch.float8_e8m0fnu]
# half a step of a rounding to the format, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -4, torch.float8_e5m2: 2.0 ** -3}
LEAST = {torch.float8_e4m3fn: 2.0 ** -9, torch.float8_e5m2: 2.0 ** -16}       # the smallest number above zero


def blocks(d):
    return -(-d // 128)


def scale_of(amax, f8, scale_dtype):
    """fp32 scale of blocks with these largest magnitudes (NaN and infinity among them)."""
    s = amax.float() / torch.full_like(amax, TOP[f8], dtype=torch.float32)
    s = torch.where(s < 2.0 ** -126, torch.full_like(s, 2.0 ** -126), s)
    if scale_dtype == torch.float32:
        return s
    m, e = torch.frexp(s)
    p = torch.ldexp(torch.ones_like(s), torch.where(m == 0.5, e - 1, e))
    return torch.where(torch.isfinite(s), p, torch.full_like(s, float("nan")))


def rows8(A, f8, scale_dtype):
    """(data, scales as fp32) of a CPU matrix."""
    n, d = A.shape
    k = blocks(d)
    x = torch.nn.functional.pad(A.float(), (0, k * 128 - d)).view(n, k, 128)
    s = scale_of(x.abs().amax(2), f8, scale_dtype)
    return (x / s[..., None]).to(f8).view(n, k * 128)[:, :d], s.t()


def weight8(W, f8, scale_dtype):
    r, c = W.shape
    kr, kc = blocks(r), blocks(c)
    x = torch.nn.functional.pad(W.float(), (0, kc * 128 - c, 0, kr * 128 - r)).view(kr, 128, kc, 128)
    s = scale_of(x.abs().amax((1, 3)), f8, scale_dtype)
    return (x / s[:, None, :, None]).to(f8).reshape(kr * 128, kc * 128)[:r, :c], s


def scale64(s):
    """Scales as numbers in 64 bits (float8_e8m0fnu: from the bytes)."""
    s = s.cpu()
    if s.dtype == torch.float32:
        return s.double()
    b = s.contiguous().view(torch.uint8).double()
    return torch.where(b == 255, torch.full_like(b, float("nan")), torch.exp2(b - 127))


def values_rows(data, scales):
    n, d = data.shape
    return data.cpu().float().double() * scale64(scales).t().repeat_interleave(128, 1)[:, :d]


def values_weight(data, scales):
    r, c = data.shape
    return data.cpu().float().double() * scale64(scales).repeat_interleave(128, 0)[:r].repeat_interleave(128, 1)[:, :c]


def bytes_of(data):
    return data.cpu().contiguous().view(torch.uint8)


def same_bytes(got, want):
    """Equal bytes; NaN may have any of its bytes."""
    got, want = got.cpu().contiguous(), want.contiguous()
    a, b = bytes_of(got), bytes_of(want)
    return bool(((a == b) | (got.float().isnan() & want.float().isnan())).all())
