"""The 8-bit operators of the RMM layer, and the norm in front of it, as cases to be timed: `listed()` names them, `draw()` gives
more of the same ranges, `prepare()` makes what a user's program holds before the call, `run()` is one pass, `work()` what a pass
cannot do without, and `exact()` the result in 64 bits.

Four ways of use ("path"):
  norm8    serving: root-mean-square norm of X (+ residual), its output in 8 bits with a scale for each 128 columns of a row
  norm     training: the norm of X (+ residual) and its backward pass
  linear8  serving: Y = X8 W8^T (+ bias), X8 with a scale for each 128 columns of a row, W8 with one for each 128 x 128 block
  step8    training: W, X and dY to 8 bits, Y = X8 W8^T and dX = dY8 W8 (the weight gradient is the sketched one of rmm_backward,
           which is not part of these operators)
Scales are fp32 numbers ("f32": amax / the format's largest value) or powers of two in 8 bits ("e8m0": the next power of two up).
Where `own` is false, `run` computes all of it from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_TOP = {"e4m3": 448.0, "e5m2": 57344.0}
_MANTISSA, _LOWEST = {"e4m3": 3, "e5m2": 2}, {"e4m3": -6, "e5m2": -14}
_SCALE = {"f32": torch.float32, "e8m0": torch.float8_e8m0fnu}
_EPS = 1e-6
_LEAST = 2.0 ** -126


def _norm8(n, d, dtype, scale, residual):
    return {"path": "norm8", "n": n, "d": d, "dtype": dtype, "scale": scale, "residual": residual}


def _norm(n, d, dtype, residual):
    return {"path": "norm", "n": n, "d": d, "dtype": dtype, "residual": residual}


def _linear8(n, d_in, d_out, out, scale, bias, f8="e4m3"):
    return {"path": "linear8", "n": n, "d_in": d_in, "d_out": d_out, "out": out, "scale": scale, "bias": bias, "f8": f8}


def _step8(n, d_in, d_out, scale, grad="e4m3"):
    return {"path": "step8", "n": n, "d_in": d_in, "d_out": d_out, "scale": scale, "grad": grad}


def listed():
    return [
        # Serving: the norm in front of a large model's projection, one new token.  Launch and latency.
        dict(_norm8(1, 1024, "bf16", "f32", True), name="norm8_token"),
        # The prompt of a base model: 8 sequences of 512 tokens.
        dict(_norm8(4096, 768, "bf16", "e8m0", True), name="norm8_prompt"),
        # fp32 activations of an odd width (no row but the first starts on 16 bytes), ragged tokens, no residual.
        dict(_norm8(1277, 1001, "f32", "f32", False), name="norm8_odd"),
        # Training step of the base model's norms.
        dict(_norm(4096, 768, "bf16", True), name="norm_base"),
        # Training at 32 sequences of 512 tokens of the large model's feed-forward width.
        dict(_norm(16384, 4096, "bf16", True), name="norm_large"),
        # Serving: one new token through the large model's feed-forward layer.  Reads the weights once.
        dict(_linear8(1, 1024, 4096, "bf16", "f32", True), name="linear8_token"),
        # A batch of 24 new tokens through its second half: a long contraction, few outputs.
        dict(_linear8(24, 4096, 1024, "bf16", "e8m0", True), name="linear8_few"),
        # Ragged tokens, widths that are no multiples of 128 or 16, fp32 result (logits).
        dict(_linear8(333, 1000, 1111, "f32", "f32", True), name="linear8_ragged"),
        # A prompt of 4096 tokens through the large model's feed-forward layer, scales as checkpoints have them.
        dict(_linear8(4096, 1024, 4096, "bf16", "f32", False), name="linear8_prompt"),
        # The largest: 16384 tokens, 4096 x 4096 weights.
        dict(_linear8(16384, 4096, 4096, "bf16", "e8m0", False), name="linear8_large"),
        # Training step of a base attention projection; gradients in the format with the wider range.
        dict(_step8(4096, 768, 768, "f32", "e5m2"), name="step8_base"),
        # Training step of the large model's feed-forward layer.
        dict(_step8(16384, 1024, 4096, "e8m0"), name="step8_large"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng):
    """Half of them multiples of 64, the others any number."""
    d = _spread(rng, 64, 4096)
    return max(64, d // 64 * 64) if rng.random() < 0.5 else d


def draw(rng):
    path = rng.choice(("norm8", "norm", "linear8", "linear8", "step8"))
    scale, half = rng.choice(("f32", "e8m0")), rng.random() < 0.5
    if path == "norm8":
        return _norm8(_spread(rng, 1, 16384), _width(rng), rng.choice(("bf16", "bf16", "f32")), scale, half)
    if path == "norm":
        return _norm(_spread(rng, 16, 16384), _width(rng), rng.choice(("bf16", "bf16", "f32")), half)
    if path == "linear8":
        return _linear8(_spread(rng, 1, 16384), _width(rng), _width(rng), rng.choice(("bf16", "bf16", "f32")), scale, half,
                        rng.choice(("e4m3", "e4m3", "e5m2")))
    return _step8(_spread(rng, 64, 8192), _width(rng), _width(rng), scale, rng.choice(("e4m3", "e5m2")))


def _blocks(d):
    return -(-d // 128)


def work(case):
    n = case["n"]
    if case["path"] in ("norm8", "norm"):
        d, size = case["d"], 2 if case["dtype"] == "bf16" else 4
        streams = 2 if case["residual"] else 1
        scales = (4 if case.get("scale") == "f32" else 1) * n * _blocks(d)
        if case["path"] == "norm8":  # X, residual, weight in; H (if there is a residual), 8-bit rows and scales out
            return {"bytes": n * d * size * (streams + (1 if case["residual"] else 0)) + d * size + n * d + scales, "flops": 8 * n * d}
        # forward: X, residual in, H, Y out; backward: dY, dH, H in, dX out; the weight and its gradient
        ways = (4 if case["residual"] else 2) + (4 if case["residual"] else 3)
        return {"bytes": n * d * size * ways + 3 * d * size + 8 * n, "flops": 20 * n * d}
    d_in, d_out = case["d_in"], case["d_out"]
    s = 4 if case["scale"] == "f32" else 1
    kin, kout = _blocks(d_in), _blocks(d_out)
    if case["path"] == "linear8":
        out = 2 if case["out"] == "bf16" else 4
        return {"bytes": n * d_in + d_out * d_in + s * (n * kin + kin * kout) + n * d_out * out + (d_out * out if case["bias"] else 0),
                "flops": 2 * n * d_in * d_out}
    # W, X and dY once in bf16 and their 8-bit forms with scales (which are results too) once, Y and dX out
    eight = n * (d_in + d_out) + d_in * d_out + s * (n * (kin + kout) + kin * kout)
    return {"bytes": 2 * (n * (d_in + d_out) + d_in * d_out) + eight + 2 * n * (d_in + d_out), "flops": 4 * n * d_in * d_out}


# ---- the plain forms: elementary operations in 32 bits


def _scale_of(amax, f8, scale):
    s = (amax / torch.full_like(amax, _TOP[f8])).clamp(min=_LEAST)  # (a quotient: a plain number would be multiplied by its inverse)
    if scale == "f32":
        return s
    m, e = torch.frexp(s)  # the next power of two, s itself where it is one
    return torch.ldexp(torch.ones_like(s), torch.where(m == 0.5, e - 1, e))


def _to8(x, s, f8):
    return (x / s).clamp(-_TOP[f8], _TOP[f8]).to(_F8[f8])


def _stored(s, scale):
    return s if scale == "f32" else s.to(torch.float8_e8m0fnu)


def _rows8(x, f8, scale):
    """x (n x d) -> its 8-bit rows, their scales (one row of n for each 128 columns)."""
    n, d = x.shape
    k = _blocks(d)
    x = torch.nn.functional.pad(x.float(), (0, k * 128 - d)).view(n, k, 128)
    s = _scale_of(x.abs().amax(2, keepdim=True), f8, scale)
    return _to8(x, s, f8).view(n, k * 128)[:, :d], s.view(n, k).t().contiguous()


def _blocks8(w, f8, scale):
    """w (rows x cols) -> its 8-bit form and a scale for each 128 x 128 block."""
    r, c = w.shape
    kr, kc = _blocks(r), _blocks(c)
    w = torch.nn.functional.pad(w.float(), (0, kc * 128 - c, 0, kr * 128 - r)).view(kr, 128, kc, 128)
    s = _scale_of(w.abs().amax((1, 3), keepdim=True), f8, scale)
    return _to8(w, s, f8).view(kr * 128, kc * 128)[:r, :c], s.view(kr, kc)


def _from_rows8(x8, s):
    n, d = x8.shape
    return x8.float() * s.t().repeat_interleave(128, 1)[:, :d]


def _from_blocks8(w8, s):
    r, c = w8.shape
    return w8.float() * s.repeat_interleave(128, 0)[:r].repeat_interleave(128, 1)[:, :c]


def _plain_norm(x, residual, weight):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    f = h.float()
    rstd = (f.square().mean(1, keepdim=True) + _EPS).rsqrt()
    return h, rstd, f * rstd * weight.float()


def _plain(state):
    case, t = state["case"], state["t"]
    path = case["path"]
    if path == "norm8":
        h, _, y = _plain_norm(t["x"], t["residual"], t["weight"])
        y8, s = _rows8(y, "e4m3", case["scale"])
        out = {"y8": y8, "scales": _stored(s, case["scale"])}
        return dict(out, h=h) if case["residual"] else out
    if path == "norm":
        h, rstd, y = _plain_norm(t["x"], t["residual"], t["weight"])
        dy, hat = t["dy"].float(), h.float() * rstd
        g = dy * t["weight"].float()
        dx = rstd * (g - hat * (g * hat).mean(1, keepdim=True))
        if case["residual"]:
            dx = dx + t["dh"].float()
        out = {"y": y.to(t["x"].dtype), "dx": dx.to(t["x"].dtype), "dweight": (dy * hat).sum(0).to(t["x"].dtype)}
        return dict(out, h=h) if case["residual"] else out
    if path == "linear8":
        s = t["x_scales"].float(), t["w_scales"].float()
        y = _from_rows8(t["x8"], s[0]) @ _from_blocks8(t["w8"], s[1]).t()
        if case["bias"]:
            y = y + t["bias"].float()
        return {"y": y.to(_DTYPE[case["out"]])}
    w8, ws = _blocks8(t["w"], "e4m3", case["scale"])
    x8, xs = _rows8(t["x"], "e4m3", case["scale"])
    g8, gs = _rows8(t["dy"], case["grad"], case["scale"])
    w = _from_blocks8(w8, ws)
    return {"y": (_from_rows8(x8, xs) @ w.t()).to(torch.bfloat16), "dx": (_from_rows8(g8, gs) @ w).to(torch.bfloat16),
            "w8": w8, "w_scales": _stored(ws, case["scale"]), "x8": x8, "x_scales": _stored(xs, case["scale"]),
            "dy8": g8, "dy_scales": _stored(gs, case["scale"])}


def _own(state):
    import paper_2201_13195_amd as rmm
    case, t = state["case"], state["t"]
    path = case["path"]
    if path == "norm8":
        r = rmm.rmm_rms_norm(t["x"], t["weight"], residual=t["residual"], eps=_EPS, need_Y=False, f8=torch.float8_e4m3fn,
                             scale_dtype=_SCALE[case["scale"]])
        out = {"y8": r.Y8, "scales": r.scales}
        return dict(out, h=r.H) if case["residual"] else out
    if path == "norm":
        r = rmm.rmm_rms_norm(t["x"], t["weight"], residual=t["residual"], eps=_EPS)
        dx, dweight = rmm.rmm_rms_norm_backward(t["dy"], r.H, t["weight"], r.rstd, dH=t["dh"])
        out = {"y": r.Y, "dx": dx, "dweight": dweight}
        return dict(out, h=r.H) if case["residual"] else out
    if path == "linear8":
        return {"y": rmm.rmm_linear8(t["x8"], t["x_scales"], t["w8"], t["w_scales"], bias=t["bias"], dtype=_DTYPE[case["out"]])}
    sd = _SCALE[case["scale"]]
    w8, ws, wt8, wts = rmm.rmm_quantize8_weight(t["w"], scale_dtype=sd, transposed=True)
    x8, xs = rmm.rmm_quantize8(t["x"], scale_dtype=sd)
    y = rmm.rmm_linear8(x8, xs, w8, ws)
    g8, gs = rmm.rmm_quantize8(t["dy"], f8=_F8[case["grad"]], scale_dtype=sd)
    return {"y": y, "dx": rmm.rmm_linear8(g8, gs, wt8, wts), "w8": w8, "w_scales": ws, "x8": x8, "x_scales": xs, "dy8": g8,
            "dy_scales": gs}


def run(state):
    return _own(state) if own else _plain(state)


# ---- inputs


def _pitched(x8):
    """The same values in rows that start on 16 bytes, which is how 8-bit matrices are kept."""
    n, d = x8.shape
    out = torch.zeros((n, (d + 15) // 16 * 16), dtype=torch.uint8, device=x8.device)
    out[:, :d] = x8.view(torch.uint8)
    return out.view(x8.dtype)[:, :d]


def _pitched_scales(s, scale):
    k, n = s.shape
    out = torch.zeros((k, (n + 15) // 16 * 16), dtype=torch.float32, device=s.device)
    out[:, :n] = s
    return _stored(out, scale)[:, :n]


def _inputs(case, seed):
    """What the operators read, from the seed alone.  Activations have a few large columns and tokens of different size, as
    those of trained models do; gradients are small and spread over orders of magnitude."""
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 17)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def acts(n, d):
        return normal(n, d) * torch.exp(0.5 * normal(n, 1)) * torch.where(normal(1, d) > 2.3, 8.0, 1.0)

    def grads(n, d):
        return normal(n, d) * torch.exp(1.5 * normal(n, 1)) * (1e-3 / math.sqrt(d))

    n = case["n"]
    if case["path"] in ("norm8", "norm"):
        d, dt = case["d"], _DTYPE[case["dtype"]]
        t = {"x": acts(n, d).to(dt), "residual": (2 * acts(n, d)).to(dt) if case["residual"] else None,
             "weight": (1 + 0.2 * normal(d)).to(dt)}
        if case["path"] == "norm":
            t["dy"], t["dh"] = grads(n, d).to(dt), grads(n, d).to(dt) if case["residual"] else None
        return t
    d_in, d_out = case["d_in"], case["d_out"]
    w = normal(d_out, d_in) * (1 / math.sqrt(d_in))
    if case["path"] == "step8":
        return {"w": w.bfloat16(), "x": acts(n, d_in).bfloat16(), "dy": grads(n, d_out).bfloat16()}
    x8, xs = _rows8(acts(n, d_in).bfloat16(), case["f8"], case["scale"])
    w8, ws = _blocks8(w.bfloat16(), "e4m3", case["scale"])
    return {"x8": _pitched(x8), "x_scales": _pitched_scales(xs, case["scale"]), "w8": _pitched(w8),
            "w_scales": _stored(ws, case["scale"]).contiguous(),
            "bias": (0.1 * normal(d_out)).to(_DTYPE[case["out"]]) if case["bias"] else None}


def prepare(case, seed):
    return {"case": case, "t": _inputs(case, seed)}


# ---- the results in 64 bits, from the definitions: an 8-bit value is q * s, s = amax / top (held in fp32) or the smallest power of
# two that is no less, no less than 2^-126 either, and q the number of the format nearest to x / s (held in fp32: with x and amax of
# few bits the quotient is often half way between two numbers of the format, and s, rounded, must not decide which)


def _nearest(v, f8):
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -40)))
    e = e + (v.abs() >= torch.exp2(e + 1)).double() - (v.abs() < torch.exp2(e)).double()
    step = torch.exp2(e.clamp(min=_LOWEST[f8]) - _MANTISSA[f8])
    return (torch.round(v / step) * step).clamp(-_TOP[f8], _TOP[f8])


def _exact_scale(amax, f8, scale):
    s = (amax / _TOP[f8]).clamp(min=_LEAST)
    if scale == "f32":
        return s.float().double()
    e = torch.ceil(torch.log2(s))
    e = e - (torch.exp2(e - 1) >= s).double() + (torch.exp2(e) < s).double()
    return torch.exp2(e)


def _exact_rows(x, f8, scale):
    q, s = torch.empty_like(x), []
    for at in range(0, x.shape[1], 128):
        part = x[:, at:at + 128]
        s.append(_exact_scale(part.abs().amax(1), f8, scale))
        q[:, at:at + 128] = _nearest((part / s[-1][:, None]).float().double(), f8)
    return q, torch.stack(s)


def _exact_blocks(w, f8, scale):
    q, s = torch.empty_like(w), torch.empty(_blocks(w.shape[0]), _blocks(w.shape[1]), dtype=torch.float64, device=w.device)
    for i in range(s.shape[0]):
        band = w[i * 128:(i + 1) * 128]
        for j in range(s.shape[1]):
            part = band[:, j * 128:(j + 1) * 128]
            s[i, j] = _exact_scale(part.abs().max(), f8, scale)
            q[i * 128:(i + 1) * 128, j * 128:(j + 1) * 128] = _nearest((part / s[i, j]).float().double(), f8)
    return q, s


def _times_rows(q, s):
    out = q.clone()
    for k in range(s.shape[0]):
        out[:, k * 128:(k + 1) * 128] *= s[k][:, None]
    return out


def _times_blocks(q, s):
    out = q.clone()
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            out[i * 128:(i + 1) * 128, j * 128:(j + 1) * 128] *= s[i, j]
    return out


def exact(case, seed):
    t = {k: v.double() if v is not None and k not in ("x_scales", "w_scales") else v for k, v in _inputs(case, seed).items()}
    path = case["path"]
    if path in ("norm8", "norm"):
        h = t["x"] if t["residual"] is None else (t["x"] + t["residual"]).to(_DTYPE[case["dtype"]]).double()
        r = 1 / torch.sqrt((h * h).sum(1, keepdim=True) / case["d"] + _EPS)
        y = h * r * t["weight"]
        if path == "norm8":
            q, s = _exact_rows(y, "e4m3", case["scale"])
            out = {"y8": q, "scales": s}
        else:
            dot = (t["dy"] * t["weight"] * h).sum(1, keepdim=True)
            dx = r * t["dy"] * t["weight"] - h * r ** 3 * dot / case["d"]
            if case["residual"]:
                dx = dx + t["dh"]
            out = {"y": y, "dx": dx, "dweight": (t["dy"] * h * r).sum(0)}
        return dict(out, h=h) if case["residual"] else out
    if path == "linear8":
        xs, ws = t["x_scales"].float().double(), t["w_scales"].float().double()
        y = _times_rows(t["x8"], xs) @ _times_blocks(t["w8"], ws).t()
        return {"y": y + t["bias"] if case["bias"] else y}
    w8, ws = _exact_blocks(t["w"], "e4m3", case["scale"])
    x8, xs = _exact_rows(t["x"], "e4m3", case["scale"])
    g8, gs = _exact_rows(t["dy"], case["grad"], case["scale"])
    w = _times_blocks(w8, ws)
    return {"y": _times_rows(x8, xs) @ w.t(), "dx": _times_rows(g8, gs) @ w, "w8": w8, "w_scales": ws, "x8": x8, "x_scales": xs,
            "dy8": g8, "dy_scales": gs}
