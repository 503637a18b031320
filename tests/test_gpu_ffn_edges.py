"""The operators around a quantized feed-forward block where rows, gates and calls are extreme, on the GPU against their formulas in
binary64 (tests/ffn_reference.py): rows whose root mean square is zero or beyond binary32, gates far out, batches of rows that lie apart in
the backward passes, large outputs over inputs."""
import pytest
import torch

import ffn_reference as R
from paper_2408_02897_amd import qmm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
FORMATS = [qmm.INT8, qmm.E4M3, qmm.E5M2]
SUM = 2.0 ** -17                                               # as in test_gpu_ffn.py: sums of a row and what follows from them


def normal(seed, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


# ------------------------------------------------------------------------------------------------ norm: no or too large a root mean square
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("cols", [3, 60, 100, 1000, 2050, 4100, 16384, 16400])
def test_norm_of_rows_without_a_root_mean_square(cols, dtype):
    """eps = 0 and rows of zeros, rows whose squares overflow, with weights that take the elements themselves past the largest value."""
    x = normal(1, 9, cols)
    x[1] = 0.0
    x[2] = -0.0
    x[3] = 2.0 ** 127                                          # times a weight of 2 or more: beyond binary32
    x[4], x[4, 0] = -2.0 ** 127, 0.0
    x[5] = 1e30                                                # only the squares are
    x[6, cols // 2] = float("inf")
    x[7, cols - 1] = float("nan")
    x = x.to(dtype)
    w = 2.0 + normal(2, cols).abs()
    for weight in (w, w.to(BF), None):
        for residual in (None, torch.zeros_like(x)):
            wd, rd = None if weight is None else weight.to(DEV), None if residual is None else residual.to(DEV)
            for fmt, mode in ((qmm.E4M3, qmm.RTNE), (qmm.INT8, qmm.RTNE), (qmm.E5M2, qmm.STOCHASTIC)):
                got = qmm.rmsnorm_quantize(x.to(DEV), wd, fmt, residual=rd, eps=0.0, mode=mode, seed=5, want_y=True, want_rstd=True)
                c, d, y, rstd = got.codes[0].cpu(), got.delta.cpu(), got.y.cpu().float(), got.rstd.cpu()
                for i in (1, 2, 3, 4, 5):
                    assert d[i] == 1 and torch.all((c[i] & 0x7F) == 0) and torch.all(y[i] == 0), i
                    assert rstd[i] == (float("inf") if i < 3 else 0.0)
                for i in (6, 7):
                    assert torch.isnan(d[i]) and torch.all(c[i] == (0 if fmt == qmm.INT8 else 0x7F)), i
                if mode == qmm.RTNE:
                    good = [0, 8]
                    R.check_codes(got.codes[0][good], got.delta[good], R.norm(x[good], None, weight, 0.0)[1], fmt, SUM)
    # weights that leave nothing of a row, and one that is no number: as the formula has it
    for weight, finite in ((torch.zeros(cols), True), (torch.full((cols,), float("inf")), False)):
        got = qmm.rmsnorm_quantize(x[[0, 3]].to(DEV), weight.to(DEV), qmm.E4M3, eps=0.0)
        assert torch.all(got.delta == 1) if finite else not torch.isfinite(got.delta).any()


def test_norm_without_columns_or_eps():
    e = qmm.rmsnorm_quantize(torch.empty((3, 0), device=DEV), None, qmm.E4M3, eps=0.0, want_rstd=True)
    assert torch.all(e.delta == 1) and torch.all(e.rstd == float("inf")) and e.codes.shape == (1, 3, 0)


# ------------------------------------------------------------------------------------------------ activations far out
# GELU: Phi(-z) = e^(-z^2/2) q(z).  In units of 2^-24, relative: q 12 (the fit 1.1, its evaluation 3.9, the argument's two roundings and reciprocal 3 times
# |t q' / q| <= 2.3) at z = 0 and falling faster than the power's constants gain, 0.023 z^2 (12.5: 6.2 + 3.6); the power 2 by the instruction and 2 by its
# correction, the product with q, that with g: 18.
PHI = 18 * 2.0 ** -24


def gates():
    return torch.cat([torch.linspace(-12.5, 12.5, 4001), torch.tensor([0.0, -0.0, 1e-30, -1e-30])])


def gated_grad_of(g, u, kind):
    """dg and du of dh = 1."""
    gu = torch.cat([g, u]).unsqueeze(0)
    v = qmm.gated_backward(torch.ones(1, g.numel(), device=DEV), gu.to(DEV), kind, want_codes=False, want_dgu=True).dgu.cpu()[0].double()
    return v[:g.numel()], v[g.numel():]


def test_gelu_keeps_its_accuracy_in_the_tail():
    g = gates()
    dg, du = gated_grad_of(g, torch.ones_like(g), qmm.GELU)
    z = g.double()
    phi, density = R.phi(z), torch.exp(-z * z / 2) * 0.3989422804014327
    assert (du - z * phi).abs().le(PHI * (z * phi).abs()).all()
    # the slope Phi + g phi(g): phi's power 4 and 3.6, its constant, a product; the sum's rounding
    assert (dg - (phi + z * density)).abs().le(PHI * phi + 10 * 2.0 ** -24 * (z * density).abs() + 2.0 ** -24 * (phi + z * density).abs()).all()
    far = torch.tensor([1e30, 3e38, 100.0, -100.0, -1e30, -3e38])
    dg, du = gated_grad_of(far, torch.ones(6), qmm.GELU)
    assert dg.tolist() == [1, 1, 1, 0, 0, 0] and du[:3].tolist() == far[:3].double().tolist() and torch.all(du[3:] == 0)
    dg, du = gated_grad_of(torch.tensor([float("nan"), float("-inf")]), torch.ones(2), qmm.GELU)
    assert torch.isnan(dg).all() and torch.isnan(du).all()


@pytest.mark.parametrize("m", [1, 100])
@pytest.mark.parametrize("kind", [qmm.SILU, qmm.GELU])
def test_product_keeps_the_stated_accuracy_in_the_tail(kind, m):
    # The header's bounds.  In units of 2^-24: the power's argument loses 1.22 of itself (the product with log2(e) and its constant; the square another 1), SiLU: the
    # instruction 2, the sum 1, the reciprocal 2, the product 1; GELU: q 12, the instruction 2, three products.
    g = torch.cat([gates()[:4000], torch.linspace(-80, 80, 4000) if kind == qmm.SILU else gates()[:4000]]).to(BF)
    f = g.numel()
    a, b = torch.zeros(m, 16, dtype=BF, device=DEV), torch.zeros(2 * f, 16, dtype=BF)
    a[:, 0], b[:f, 0], b[f:, 0] = 1.0, g, 1.0
    b = b.to(DEV)
    h = qmm.gemm_gated((a, qmm.operand(a, qmm.BF16, is_codes=False)), (b, qmm.operand(b, qmm.BF16, is_codes=False)), kind, F32)[0].cpu().double()
    z = g.double()
    want = R.act(z, kind)[0]
    off = (1.3 * z.abs() + 8 if kind == qmm.SILU else 1.2 * z * z + 18) * 2.0 ** -24
    assert ((h - want).abs() <= off * want.abs()).all()


def test_silu_slope_keeps_its_accuracy():
    # s (1 + g (1 - s)), in units of 2^-24: s 5 (see test_logistic_keeps_its_accuracy_in_the_tail: power 3, sum, last step), 1 - s as e^-g s 3 + 5 + 1,
    # the sum's and the product's rounding, 1 for what is of second order
    g = torch.cat([torch.linspace(-79.9, 79.9, 20001), torch.linspace(0, 20, 20001), torch.tensor([0.0, -0.0, 1e-30, -1e-30])])
    dg, _ = gated_grad_of(g, torch.ones_like(g), qmm.SILU)
    z = g.double()
    s, rest = torch.sigmoid(z), torch.sigmoid(-z)
    assert (dg - s * (1 + z * rest)).abs().le(2.0 ** -24 * s * (8 * (1 + z * rest).abs() + 9 * (z * rest).abs())).all()
    far = torch.tensor([1e30, 3e38, 100.0, -100.0, -1e30, -3e38])
    dg, _ = gated_grad_of(far, torch.ones(6), qmm.SILU)
    assert dg[:3].tolist() == [1, 1, 1] and dg[3:].abs().le(1e-30).all()


# ------------------------------------------------------------------------------------------------ backward passes of batches
def apart(t, rows, cols):
    """The same batch with `rows` rows between the matrices and `cols` elements between the rows, filled with NaN, off a 16-byte boundary."""
    b, r, c = t.shape
    big = torch.full((b * (r + rows) * (c + cols) + 1,), float("nan"), dtype=t.dtype, device=DEV)[1:].view(b, r + rows, c + cols)
    v = big[:, :r, :c]
    v.copy_(t)
    return v


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", [(7, 30), (11, 100), (401, 64), (5, 1000), (9, 4104), (3, 16400)])
def test_norm_backward_of_batches(rows, cols, dtype):
    dy, h, r = normal(1, 3, rows, cols, dtype=dtype, scale=0.01), normal(2, 3, rows, cols, dtype=dtype, scale=2.0), normal(3, 3, rows, cols, dtype=dtype, scale=0.01)
    w = 1 + 0.3 * normal(4, cols)
    rstd = R.norm(h, None, None, 1e-5)[2].float()
    dx, dw, size, size_w = R.norm_grad(dy, h, rstd, w, r)
    for args in ((dy.to(DEV), h.to(DEV), r.to(DEV)), (apart(dy, 2, 3), apart(h, 1, 0), apart(r, 0, 5))):
        gx, gw = qmm.rmsnorm_backward(args[0], args[1], rstd.reshape(-1).to(DEV), w.to(DEV), dresidual=args[2])
        assert gx.shape == dy.shape
        assert ((gx.cpu().double() - dx).abs() <= SUM * size + R.rounding(dtype) * dx.abs()).all()
        assert ((gw.cpu().double() - dw).abs() <= SUM * size_w).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,f", [(7, 30), (11, 100), (5, 1000), (9, 4104), (3, 16400)])
def test_gated_backward_of_batches(rows, f, dtype):
    dh, gu = normal(1, 3, rows, f, dtype=dtype), normal(2, 3, rows, 2 * f, dtype=dtype, scale=1.5)
    g, u, d = gu[..., :f].double(), gu[..., f:].double(), dh.double()
    for kind in (qmm.SILU, qmm.GELU):
        value, slope = R.act(g, kind)
        want = torch.cat([d * u * slope, d * value], -1)
        # |g| <= 8 here: the terms of the slope, relative to 32 roundings each (the tests above)
        terms = torch.cat([(d * u).abs() * (1 + g.abs()), (d * value).abs()], -1)
        for args in ((dh.to(DEV), gu.to(DEV)), (apart(dh, 2, 3), apart(gu, 1, 5))):
            got = qmm.gated_backward(*args, kind, qmm.E5M2, want_dgu=True)
            assert got.dgu.shape == gu.shape and got.codes.shape == gu.shape
            off = 32 * 2.0 ** -24 * terms
            assert ((got.dgu.cpu().double() - want).abs() <= off + R.rounding(dtype) * (want.abs() + off)).all()
            R.check_codes(got.codes, got.delta, want, qmm.E5M2, 2.0 ** -14)


# ------------------------------------------------------------------------------------------------ large outputs over inputs
def test_large_outputs_over_inputs():
    """From 64 MB on rows are read and written past the caches: the same results where an output takes an input's memory."""
    rows, cols = 8192, 4096
    g = torch.Generator(device=DEV).manual_seed(3)
    x, r = (torch.randn((rows, cols), generator=g, device=DEV, dtype=BF) for _ in range(2))
    w = torch.rand(cols, generator=g, device=DEV) + 0.5
    n = qmm.rmsnorm_quantize(x, w, qmm.E4M3, residual=r, want_y=True, want_rstd=True)
    for which in range(2):
        t = [x.clone(), r.clone()]
        m = qmm.rmsnorm_quantize(t[0], w, qmm.E4M3, residual=t[1], want_y=True, want_rstd=True, h_out=t[which])
        assert m.h is t[which] and all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(n, m))
    dx, dw = qmm.rmsnorm_backward(n.y, n.h, n.rstd, w, dresidual=r)
    for which in range(3):
        t = [n.y.clone(), n.h.clone(), r.clone()]
        dx2, dw2 = qmm.rmsnorm_backward(t[0], t[1], n.rstd, w, dresidual=t[2], dx_out=t[which])
        assert dx2 is t[which] and torch.equal(dx, dx2) and torch.equal(dw, dw2)
    gu = torch.randn((rows, 2 * cols), generator=g, device=DEV, dtype=BF)
    d = qmm.gated_backward(x, gu, qmm.SILU, qmm.E5M2, want_dgu=True)
    e = qmm.gated_backward(x, gu, qmm.SILU, qmm.E5M2, dgu_out=gu)
    assert e.dgu is gu and torch.equal(d.dgu, gu) and torch.equal(d.codes, e.codes) and torch.equal(d.delta, e.delta)


# ------------------------------------------------------------------------------------------------ operands
def test_gated_product_refuses_operands_that_read_past_their_tensors(monkeypatch):
    x, w = torch.zeros((4, 32), dtype=torch.uint8, device=DEV), torch.zeros((20, 32), dtype=torch.uint8, device=DEV)
    op = lambda t, n, **k: (t, qmm.operand(t, qmm.E4M3, torch.ones(n, device=DEV), **k))
    a, b = op(x, 4, per_channel=True), op(w, 20, per_channel=True)
    for short in (None, qmm._NoShortPath):
        monkeypatch.setattr(qmm, "_short", short)
        for good in ((a, b), (op(x, 1), b), (op(x, 7, per_channel=True), op(w, 2))):
            assert torch.all(qmm.gemm_gated(*good) == 0)
        for bad in ((op(x, 3, per_channel=True), b), (a, op(w, 10, per_channel=True)), (a, (torch.zeros_like(w), b[1])), (op(x.to(BF), 4, per_channel=True), b),
                    (a, (w, qmm.operand(w, qmm.E4M3, torch.ones(20), per_channel=True)))):
            with pytest.raises(ValueError):
                qmm.gemm_gated(*bad)
