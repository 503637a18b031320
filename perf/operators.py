"""The operators around a quantized feed-forward block, as cases that can be timed and compared:

  norm       residual addition, root-mean-square norm and 8-bit codes with one step size per token (qmm.rmsnorm_quantize)
  norm_grad  its backward pass (qmm.rmsnorm_backward)
  gated      both projections of a gated feed-forward block, the activation and the product (qmm.gemm_gated)
  gated_grad its backward pass up to the operand of the products that follow (qmm.gated_backward)

With `own` false a case runs in plain torch operations in binary32 (sums over many rows in binary64), rounded once at the end."""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-6
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
QMAX = {"int8": 127.0, "e4m3": 448.0, "e5m2": 57344.0}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
GRID = {"e4m3": (3, -6), "e5m2": (2, -14)}          # mantissa bits, exponent of the smallest normal value


def listed():
    return [
        # one token being generated: what counts is latency
        dict(name="norm one token", kind="norm", rows=1, cols=4096, src="bf16", fmt="e4m3", residual=True, train=False),
        # a ragged batch of a float32 model, no residual (the first norm of a stack), INT8
        dict(name="norm ragged int8", kind="norm", rows=1031, cols=1000, src="f32", fmt="int8", residual=False, train=False),
        # a training step's tokens (batch 32 x 512); normalised values and 1 / rms are kept for the backward pass
        dict(name="norm training", kind="norm", rows=16384, cols=4096, src="bf16", fmt="e4m3", residual=True, train=True),
        # backward passes of the last two
        dict(name="norm grad ragged f32", kind="norm_grad", rows=1031, cols=1000, src="f32", residual=False),
        dict(name="norm grad training", kind="norm_grad", rows=16384, cols=4096, src="bf16", residual=True),
        # one token being generated: the weights are read once
        dict(name="gated one token", kind="gated", m=1, f=8192, k=4096, fmt="e4m3", fmt_b="e4m3", act="silu", out="bf16", train=False),
        # a few sequences decoded together, INT8
        dict(name="gated 24 tokens int8", kind="gated", m=24, f=4096, k=1024, fmt="int8", fmt_b="int8", act="silu", out="bf16", train=False),
        # a prompt of odd length through a narrow model without quantization (the high-precision side of a comparison)
        dict(name="gated prompt bf16", kind="gated", m=1031, f=2000, k=784, fmt="bf16", fmt_b="bf16", act="gelu", out="f32", train=False),
        # a whole batch without a backward pass to come (evaluation), INT8
        dict(name="gated batch int8", kind="gated", m=4096, f=2048, k=768, fmt="int8", fmt_b="int8", act="gelu", out="bf16", train=False),
        # a training step's tokens; both projections are kept for the backward pass
        dict(name="gated training", kind="gated", m=16384, f=4096, k=1024, fmt="e4m3", fmt_b="e4m3", act="silu", out="bf16", train=True),
        # backward passes
        dict(name="gated grad ragged f32", kind="gated_grad", m=257, f=1000, src="f32", fmt="e5m2", act="gelu"),
        dict(name="gated grad training", kind="gated_grad", m=16384, f=4096, src="bf16", fmt="e5m2", act="silu"),
    ]


def _log(rng, lo, hi, of=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / of)) * of))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "gated", "gated_grad"])
    if kind == "gated":
        k, f = _log(rng, 64, 8192, 16), _log(rng, 64, 8192)
        m = _log(rng, 1, max(1, min(16384, (1 << 36) // (k * f))))
        fmt = rng.choice(["int8", "e4m3", "e5m2", "bf16"])
        fmt_b = rng.choice(["e4m3", "e5m2"]) if fmt in FLOAT8 else fmt
        return dict(kind=kind, m=m, f=f, k=k, fmt=fmt, fmt_b=fmt_b, act=rng.choice(["silu", "gelu"]), out=rng.choice(["bf16", "f32"]), train=rng.random() < 0.5)
    cols = _log(rng, 64, 8192)
    rows = _log(rng, 1, min(16384, (1 << 25) // cols if kind == "gated_grad" else (1 << 26) // cols))
    src = rng.choice(["bf16", "f32"])
    if kind == "norm":
        return dict(kind=kind, rows=rows, cols=cols, src=src, fmt=rng.choice(["int8", "e4m3", "e5m2"]), residual=rng.random() < 0.7, train=rng.random() < 0.5)
    if kind == "norm_grad":
        return dict(kind=kind, rows=rows, cols=cols, src=src, residual=rng.random() < 0.7)
    return dict(kind=kind, m=rows, f=cols, src=src, fmt=rng.choice(["int8", "e4m3", "e5m2"]), act=rng.choice(["silu", "gelu"]))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def gradient(*shape):                        # signs and log-normal magnitudes, as upstream gradients have them
        return torch.exp(2.0 * normal(*shape) - 8.0) * torch.where(normal(*shape) < 0, -1.0, 1.0)

    def coded(v, fmt):                           # codes and one step size per row
        if fmt == "bf16":
            return v.to(torch.bfloat16), None
        d = (v.abs().amax(1) / QMAX[fmt]).clamp_min(2.0 ** -126)
        t = (v / d[:, None]).clamp(-QMAX[fmt], QMAX[fmt])
        return (t.round().to(torch.int8) if fmt == "int8" else t.to(FLOAT8[fmt])).view(torch.uint8), d

    s = dict(case=case)
    if case["kind"] == "gated":
        m, f, k = case["m"], case["f"], case["k"]
        s["a"], s["da"] = coded(normal(m, k), case["fmt"])
        s["w"], s["dw"] = coded(normal(2 * f, k) * (1.5 / math.sqrt(k)), case["fmt_b"])
        return s
    dt = DTYPE[case["src"]]
    if case["kind"] == "gated_grad":
        s["dh"], s["gu"] = gradient(case["m"], case["f"]).to(dt), (1.5 * normal(case["m"], 2 * case["f"])).to(dt)
        return s
    rows, cols = case["rows"], case["cols"]
    s["weight"] = (1.0 + 0.2 * normal(cols)).to(dt)
    s["x"] = (normal(rows, cols) * torch.exp(0.5 * normal(1, cols))).to(dt)       # some channels larger than others
    s["residual"] = (2.0 * normal(rows, cols)).to(dt) if case["residual"] else None
    if case["kind"] == "norm_grad":
        s["dy"] = gradient(rows, cols).to(dt)
        s["residual"] = gradient(rows, cols).to(dt) if case["residual"] else None
        s["rstd"] = torch.rsqrt(s["x"].double().square().mean(1) + EPS).float()
    return s


def _quantized(y, fmt):
    """Codes of the rows of y (binary32) as the values they stand for, and the step sizes."""
    d = y.abs().amax(1) / QMAX[fmt]
    d = torch.where(d == 0, 1.0, d.clamp_min(2.0 ** -126))
    t = (y * (1.0 / d)[:, None]).clamp(-QMAX[fmt], QMAX[fmt])
    if fmt == "int8":
        return (t.round() * d[:, None]).to(torch.bfloat16), d
    return t.to(FLOAT8[fmt]), d


def _values(codes, fmt, delta):
    """The same of codes that the framework wrote: FP8 bytes as they are, INT8 times the step size."""
    from paper_2408_02897_amd import qmm
    if fmt == "int8":
        return qmm.dequantize(codes, qmm.INT8, delta, per_channel=True, out_dtype=torch.bfloat16)[0]
    return codes[0].view(FLOAT8[fmt])


def _plain_norm(s):
    c = s["case"]
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    v = h.float()
    rstd = torch.rsqrt((v * v).mean(1) + EPS)
    y = v * rstd[:, None] * s["weight"].float()
    out = dict(zip(("codes", "delta"), _quantized(y, c["fmt"])))
    if s["residual"] is not None:
        out["h"] = h
    if c["train"]:
        out["y"], out["rstd"] = y.to(h.dtype), rstd
    return out


def _plain_norm_grad(s):
    dt = s["x"].dtype
    dy, xhat = s["dy"].float(), s["x"].float() * s["rstd"][:, None]
    a = dy * s["weight"].float()
    dx = s["rstd"][:, None] * (a - xhat * (a * xhat).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dict(dx=dx.to(dt), dw=(dy * xhat).sum(0, dtype=torch.float64).float())


def _decoded(codes, d, fmt):
    if fmt == "bf16":
        return codes.float()
    v = codes.view(torch.int8) if fmt == "int8" else codes.view(FLOAT8[fmt])
    return v.float() * d[:, None]


def _plain_gated(s):
    c = s["case"]
    gu = _decoded(s["a"], s["da"], c["fmt"]) @ _decoded(s["w"], s["dw"], c["fmt_b"]).t()
    g, u = gu[:, :c["f"]], gu[:, c["f"]:]
    act = g / (1.0 + torch.exp(-g)) if c["act"] == "silu" else 0.5 * g * (1.0 + torch.erf(g * math.sqrt(0.5)))
    dt = DTYPE[c["out"]]
    return dict(h=(act * u).to(dt), **(dict(gu=gu.to(dt)) if c["train"] else {}))


def _plain_gated_grad(s):
    c = s["case"]
    dh, g, u = s["dh"].float(), s["gu"][:, :c["f"]].float(), s["gu"][:, c["f"]:].float()
    if c["act"] == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        slope = p * (1.0 + g * (1.0 - p))
    else:
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        slope = p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    d = torch.cat([dh * u * slope, dh * g * p], 1)
    return dict(zip(("codes", "delta"), _quantized(d, c["fmt"])), dgu=d.to(s["dh"].dtype))


def _own(s):
    from paper_2408_02897_amd import qmm
    c = s["case"]
    fmt = {"int8": qmm.INT8, "e4m3": qmm.E4M3, "e5m2": qmm.E5M2, "bf16": qmm.BF16}
    act = {"silu": qmm.SILU, "gelu": qmm.GELU}
    if c["kind"] == "norm":
        r = qmm.rmsnorm_quantize(s["x"], s["weight"], fmt[c["fmt"]], residual=s["residual"], eps=EPS, want_y=c["train"], want_rstd=c["train"])
        out = dict(codes=_values(r.codes, c["fmt"], r.delta), delta=r.delta)
        if s["residual"] is not None:
            out["h"] = r.h
        if c["train"]:
            out["y"], out["rstd"] = r.y, r.rstd
        return out
    if c["kind"] == "norm_grad":
        dx, dw = qmm.rmsnorm_backward(s["dy"], s["x"], s["rstd"], s["weight"], dresidual=s["residual"])
        return dict(dx=dx, dw=dw)
    if c["kind"] == "gated":
        quantized = c["fmt"] != "bf16"
        a = (s["a"], qmm.operand(s["a"], fmt[c["fmt"]], s["da"], per_channel=quantized, is_codes=quantized))
        w = (s["w"], qmm.operand(s["w"], fmt[c["fmt_b"]], s["dw"], per_channel=quantized, is_codes=quantized))
        r = qmm.gemm_gated(a, w, act[c["act"]], DTYPE[c["out"]], want_gu=c["train"])
        return dict(h=r[0][0], gu=r[1][0]) if c["train"] else dict(h=r[0])
    r = qmm.gated_backward(s["dh"], s["gu"], act[c["act"]], fmt[c["fmt"]], want_dgu=True)
    return dict(codes=_values(r.codes, c["fmt"], r.delta), delta=r.delta, dgu=r.dgu)


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "gated": _plain_gated, "gated_grad": _plain_gated_grad}[state["case"]["kind"]](state)


def work(case):
    if case["kind"] == "gated":
        m, f, k = case["m"], case["f"], case["k"]
        es, eo = 2 if case["fmt"] == "bf16" else 1, 2 if case["out"] == "bf16" else 4
        steps = 0 if case["fmt"] == "bf16" else 4 * (m + 2 * f)
        return dict(bytes=(m + 2 * f) * k * es + steps + m * f * eo * (3 if case["train"] else 1), flops=4 * m * f * k)
    e = 2 if case["src"] == "bf16" else 4
    if case["kind"] == "gated_grad":
        n = case["m"] * case["f"]
        return dict(bytes=n * (3 * e + 2 + 2 * e) + 4 * case["m"], flops=20 * n)
    n, rows, cols = case["rows"] * case["cols"], case["rows"], case["cols"]
    if case["kind"] == "norm":
        per = e + 1 + (2 * e if case["residual"] else 0) + (e if case["train"] else 0)
        return dict(bytes=n * per + cols * e + 4 * rows * (2 if case["train"] else 1), flops=10 * n)
    return dict(bytes=n * e * (4 if case["residual"] else 3) + cols * (e + 4) + 4 * rows, flops=12 * n)


def _nearest(t, fmt):
    """The value of the format's grid nearest to t (binary64), ties to the even one, saturating."""
    t = t.clamp(-QMAX[fmt], QMAX[fmt])
    if fmt == "int8":
        return torch.round(t)
    bits, least = GRID[fmt]
    e = torch.clamp(torch.frexp(t)[1].double() - 1, min=float(least)) - bits
    return (torch.ldexp(torch.round(torch.ldexp(t, -e)), e)).clamp(-QMAX[fmt], QMAX[fmt])


def _exact_codes(v, fmt):
    delta = torch.max(torch.abs(v), dim=1).values / QMAX[fmt]
    delta = torch.where(delta > 0, torch.clamp(delta, min=2.0 ** -126), torch.ones_like(delta))
    q = _nearest(v / delta.unsqueeze(1), fmt)
    return (q * delta.unsqueeze(1) if fmt == "int8" else q), delta


def _normal_cdf(g):
    return 0.5 * torch.special.erfc(-g / math.sqrt(2.0))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "gated":
        fmts, ops = (case["fmt"], case["fmt_b"]), []
        for codes, d, fmt in zip((s["a"], s["w"]), (s["da"], s["dw"]), fmts):
            v = codes if fmt == "bf16" else codes.view(torch.int8 if fmt == "int8" else FLOAT8[fmt])
            ops.append(v.double() if d is None else v.double().mul_(d.double().unsqueeze(1)))
        gate = torch.mm(ops[0], ops[1][:case["f"]].t().contiguous())
        up = torch.mm(ops[0], ops[1][case["f"]:].t().contiguous())
        a = gate * torch.sigmoid(gate) if case["act"] == "silu" else gate * _normal_cdf(gate)
        out = dict(h=a.mul_(up))
        if case["train"]:
            out["gu"] = torch.cat([gate, up], dim=1)
        return out
    if case["kind"] == "gated_grad":
        gate, up = torch.split(s["gu"].double(), case["f"], dim=1)
        if case["act"] == "silu":
            sig = torch.sigmoid(gate)
            value, slope = gate * sig, sig + gate * sig * torch.sigmoid(-gate)
        else:
            value, slope = gate * _normal_cdf(gate), _normal_cdf(gate) + gate * torch.exp(-gate.square() / 2) / math.sqrt(2 * math.pi)
        v = torch.cat([s["dh"].double() * up * slope, s["dh"].double() * value], dim=1)
        codes, delta = _exact_codes(v, case["fmt"])
        return dict(codes=codes, delta=delta, dgu=v)
    w = s["weight"].double()
    if case["kind"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:               # the sum as it is stored is what is normalised
            h = (h + s["residual"].double()).to(DTYPE[case["src"]]).double()
        rstd = 1.0 / torch.sqrt(h.square().mean(dim=1) + EPS)
        y = h * rstd.unsqueeze(1) * w
        codes, delta = _exact_codes(y, case["fmt"])
        out = dict(codes=codes, delta=delta)
        if s["residual"] is not None:
            out["h"] = h
        return out | (dict(y=y, rstd=rstd) if case["train"] else {})
    dy, n, r = s["dy"].double(), s["x"].double() * s["rstd"].double().unsqueeze(1), s["rstd"].double().unsqueeze(1)
    dx = r * (w * dy - n * (w * dy * n).sum(dim=1, keepdim=True) / case["cols"])
    if s["residual"] is not None:
        dx = dx + s["residual"].double()
    return dict(dx=dx, dw=(dy * n).sum(dim=0))
