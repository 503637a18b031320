"""The gradients of tests/ffn_reference.py against differences of its own forward formulas, and the refusals of the operators
that it stands for, all on the host."""
import ctypes
import os

import pytest
import torch

import ffn_reference as R
from paper_2408_02897_amd import qmm


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qmm.LIB_PATH):
        from paper_2408_02897_amd import build
        build.build()
    return qmm.lib()


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("residual", [False, True])
def test_norm_gradient_is_that_of_the_formula(residual):
    x, w, dy, v = _normal(1, 5, 33), _normal(2, 33), _normal(3, 5, 33), _normal(4, 5, 33)
    past = _normal(5, 5, 33) if residual else None
    eps, step = 1e-3, 1e-6

    def loss(x, w):                                            # (x is binary64: no rounding of the sum)
        y = R.norm(x, None, w, eps)[1]
        return (y * dy).sum() + (0 if past is None else (x * past).sum())
    dx, dw, _, _ = R.norm_grad(dy, x, R.norm(x, None, w, eps)[2], w, past)
    # central differences: the third derivative's part is of the order step^2, rounding 2^-52 |loss| / step: both below 1e-8
    assert abs((loss(x + step * v, w) - loss(x - step * v, w)) / (2 * step) - (dx * v).sum()) < 1e-7
    u = _normal(6, 33)
    assert abs((loss(x, w + step * u) - loss(x, w - step * u)) / (2 * step) - (dw * u).sum()) < 1e-7


@pytest.mark.parametrize("kind", [0, 1])
def test_activation_slopes_are_those_of_the_formulas(kind):
    g = torch.linspace(-12, 12, 4001, dtype=torch.float64)
    step = 1e-5                                                # third derivatives are below 2: step^2 / 6 of that; rounding 2^-52 * 12 / step
    diff = (R.act(g + step, kind)[0] - R.act(g - step, kind)[0]) / (2 * step)
    assert (diff - R.act(g, kind)[1]).abs().max() < 1e-9


def test_norm_refusals(L):
    p, off = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10002)
    T = lambda **k: qmm.Tensor(*{**dict(data=0x20000, dtype=qmm.DT_F32, axis=1, b=2, r=4, c=16, bs=64, rs=16), **k}.values())
    ref = ctypes.byref

    def fwd(x, r=None, w=p, wt=qmm.DT_F32, eps=1e-6, fmt=qmm.E4M3, mode=0, h=None, y=None, rstd=None, d=p, c=p):
        return L.qmm_rmsnorm_quantize(None if x is None else ref(x), None if r is None else ref(r), w, wt, eps, fmt, mode, 0, 0, h, y, rstd, d, c, None)
    assert fwd(None) == 1 and fwd(T(), d=None) == 1 and fwd(T(), c=None) == 1 and fwd(T(data=None)) == 1
    assert fwd(T(), T(), h=None) == 1 and fwd(T(), T(data=None), h=p) == 1
    assert fwd(T(dtype=5)) == 3 and fwd(T(axis=7)) == 3 and fwd(T(axis=0)) == 5
    assert fwd(T(), wt=9) == 3 and fwd(T(), fmt=3) == 3 and fwd(T(), fmt=-1) == 3 and fwd(T(), mode=2) == 3
    assert fwd(T(c=-1)) == 2 and fwd(T(rs=8)) == 2 and fwd(T(bs=10)) == 2 and fwd(T(r=-3)) == 2
    assert fwd(T(b=65536)) == 5 and fwd(T(b=1, r=1, c=(1 << 22) + 1, rs=1 << 23)) == 5
    assert fwd(T(), T(c=8, rs=16), h=p) == 2 and fwd(T(), T(r=3), h=p) == 2 and fwd(T(), T(dtype=qmm.DT_BF16), h=p) == 5
    for eps in (-1.0, float("nan"), float("inf")):
        assert fwd(T(), eps=eps) == 2
    for k in ("w", "h", "y", "rstd", "d"):
        assert fwd(T(), T(), **{**dict(h=p), k: off}) == 4
    assert fwd(T(data=0x20002)) == 4
    assert fwd(T(rs=20, bs=80), T(), h=ctypes.c_void_p(0x20000)) == 2           # over an input whose rows lie apart
    assert fwd(T(), T(data=0x30000), h=p, y=p) == 2
    assert fwd(T(b=0), d=None, c=None) == 0 and fwd(T(r=0, data=None), d=None, c=None) == 0

    assert L.qmm_rmsnorm_backward_workspace_size(ref(T())) == 0                   # few rows: one share, which is dw
    many = dict(r=400, bs=6400)
    need = L.qmm_rmsnorm_backward_workspace_size(ref(T(**many)))
    assert need > 0 and need % 64 == 0 and L.qmm_rmsnorm_backward_workspace_size(ref(T(rs=8))) == 0 and L.qmm_rmsnorm_backward_workspace_size(None) == 0

    def bwd(dy, h, r=None, rstd=p, w=p, wt=qmm.DT_F32, dx=p, dw=p, ws=p, nws=1 << 20):
        return L.qmm_rmsnorm_backward(None if dy is None else ref(dy), None if h is None else ref(h), rstd, w, wt, None if r is None else ref(r), dx, dw, ws, nws, None)
    assert bwd(None, T()) == 1 and bwd(T(), None) == 1 and bwd(T(), T(), rstd=None) == 1 and bwd(T(), T(), dx=None) == 1
    assert bwd(T(data=None), T()) == 1 and bwd(T(), T(data=None)) == 1 and bwd(T(), T(), T(data=None)) == 1
    assert bwd(T(), T(c=8)) == 2 and bwd(T(), T(), T(r=5, bs=80)) == 2 and bwd(T(), T(dtype=qmm.DT_BF16)) == 5 and bwd(T(), T(axis=0)) == 5
    assert bwd(T(), T(), wt=4) == 3 and bwd(T(), T(), rstd=off) == 4 and bwd(T(), T(), dw=off) == 4 and bwd(T(), T(), dx=off) == 4
    assert bwd(T(**many), T(**many), ws=None) == 6 and bwd(T(**many), T(**many), nws=need - 1) == 6 and bwd(T(**many), T(**many), ws=ctypes.c_void_p(0x10004)) == 4
    assert bwd(T(rs=20, bs=80), T(), dx=ctypes.c_void_p(0x20000)) == 2
    assert bwd(T(c=0, rs=0), T(c=0, rs=0)) == 0


def test_gated_refusals(L):
    p, off = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)
    ref, g = ctypes.byref, qmm.granularity(True, 1)
    O = lambda fmt=qmm.E4M3, codes=1, data=p, delta=p, gran=g: qmm.Operand(data, fmt, codes, delta, gran)

    def run(a, b, n=(1, 8, 16, 32), act=0, h=p, gu=None, out=0, ws=None, nws=0):
        return L.qmm_gemm_gated(None if a is None else ref(a), None if b is None else ref(b), *n, act, h, gu, out, ws, nws, None)
    assert run(None, O()) == 1 and run(O(), None) == 1 and run(O(), O(), h=None) == 1
    assert run(O(delta=None), O()) == 1 and run(O(), O(delta=None)) == 1 and run(O(data=None), O()) == 1
    assert run(O(fmt=9), O()) == 3 and run(O(), O(codes=2)) == 3 and run(O(), O(), act=2) == 3 and run(O(), O(), act=-1) == 3 and run(O(), O(), out=7) == 3
    assert run(O(), O(gran=qmm.granularity(True, 0))) == 3
    assert run(O(), O(fmt=qmm.INT8)) == 5 and run(O(), O(fmt=qmm.BF16, codes=0)) == 5 and run(O(codes=0), O()) == 5 and run(O(), O(codes=0)) == 5
    assert run(O(), O(), n=(1, -8, 16, 32)) == 2 and run(O(), O(), n=(1, 8, -1, 32)) == 2 and run(O(), O(), n=(-1, 8, 16, 32)) == 2
    assert run(O(), O(), n=(1, 8, 16, 24)) == 4 and run(O(data=off), O()) == 4 and run(O(), O(), h=off) == 4 and run(O(), O(), gu=off) == 4
    assert run(O(), O(), n=(1, 8, 16, (1 << 22) + 16)) == 5 and run(O(), O(), n=(1, 8, (1 << 22) + 1, 32)) == 5
    for n in ((0, 8, 16, 32), (1, 0, 16, 32), (1, 8, 0, 32)):
        assert run(O(data=None), O(), n=n, h=None) == 0 and L.qmm_gemm_gated_workspace_size(ref(O()), ref(O()), *n) == 0
    assert L.qmm_gemm_gated_workspace_size(None, ref(O()), 1, 8, 16, 32) == 0
    # few columns and a long contraction: split, with a workspace for the parts
    for n in ((1, 8, 64, 8192), (1, 200, 100, 4096), (2, 64, 16, 6144)):
        need = L.qmm_gemm_gated_workspace_size(ref(O()), ref(O()), *n)
        assert need > 0 and need % (8 * n[0] * n[1] * n[2]) == 0
        assert run(O(), O(), n=n) == 6 and run(O(), O(), n=n, ws=p, nws=need - 1) == 6 and run(O(), O(), n=n, ws=ctypes.c_void_p(0x10004), nws=need) == 4

    T = lambda **k: qmm.Tensor(*{**dict(data=0x20000, dtype=qmm.DT_F32, axis=1, b=2, r=4, c=16, bs=128, rs=32), **k}.values())

    def bwd(dh, gu, act=0, fmt=qmm.E5M2, mode=0, dgu=None, d=p, c=p):
        return L.qmm_gated_backward(None if dh is None else ref(dh), None if gu is None else ref(gu), act, fmt, mode, 0, 0, dgu, d, c, None)
    G = lambda **k: T(**{**dict(c=32), **k})
    assert bwd(None, G()) == 1 and bwd(T(), None) == 1 and bwd(T(), G(), d=None) == 1 and bwd(T(), G(), c=None) == 1 and bwd(T(), G(), d=None, c=None) == 1
    assert bwd(T(data=None), G()) == 1 and bwd(T(), G(data=None)) == 1
    assert bwd(T(), T()) == 2 and bwd(T(), G(r=3)) == 2 and bwd(T(b=1), G()) == 2 and bwd(T(rs=8), G()) == 2
    assert bwd(T(), G(dtype=qmm.DT_BF16)) == 5 and bwd(T(), G(axis=0)) == 5
    assert bwd(T(), G(), act=2) == 3 and bwd(T(), G(), fmt=3) == 3 and bwd(T(), G(), mode=2) == 3
    assert bwd(T(), G(), d=ctypes.c_void_p(0x10002)) == 4 and bwd(T(), G(), dgu=ctypes.c_void_p(0x10002)) == 4 and bwd(T(data=0x20001), G()) == 4
    assert bwd(T(), G(data=0x30000), dgu=ctypes.c_void_p(0x20000)) == 2                           # over dh
    assert bwd(T(data=0x30000), G(rs=40, bs=160), dgu=ctypes.c_void_p(0x20000)) == 2             # over rows that lie apart
    assert bwd(T(b=0), G(b=0)) == 0 and bwd(T(r=0), G(r=0), d=None, c=None, dgu=p) == 0


def test_the_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros((4, 32))
    for call in (lambda: qmm.rmsnorm_quantize(x, None, qmm.E4M3), lambda: qmm.rmsnorm_backward(x, x, x[:, 0], None), lambda: qmm.gated_backward(x, x)):
        with pytest.raises(ValueError):                        # not on a GPU
            call()
    op = qmm.operand(torch.zeros((4, 32), dtype=torch.uint8), qmm.E4M3, torch.ones(1))
    with pytest.raises(ValueError):
        qmm.gemm_gated((x, op), (x, op))


def test_gated_product_refuses_operands_that_read_past_their_tensors(monkeypatch):
    """Step sizes or elements that are not there: refused before the library is called (the kernels read what the descriptor says)."""
    class Reached(Exception):
        pass

    class Library:
        def __getattr__(self, name):
            if "workspace" in name:
                return lambda *_: 0
            raise Reached(name)
    monkeypatch.setattr(qmm, "_on", lambda device, *tensors: device)
    monkeypatch.setattr(qmm, "lib", Library)
    monkeypatch.setattr(qmm, "_short", qmm._NoShortPath)
    codes = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    x, w = codes(4, 32), codes(20, 32)
    op = lambda t, n, fmt=qmm.E4M3, **k: (t, qmm.operand(t, fmt, torch.ones(n), **k))
    whole = op(x, 4, per_channel=True), op(w, 20, per_channel=True)
    good = [whole, (op(x, 1), op(w, 1)), (op(x, 9, per_channel=True), op(w, 3)),
            (op(codes(6, 4, 32), 3 * 4, per_channel=True, batch_groups=3), op(codes(6, 20, 32), 2, batch_groups=2, batch_inner=3)),
            (op(codes(2, 4, 32), 4 * 2, per_channel=True, batch_groups=5), op(codes(2, 20, 32), 1, batch_groups=4, batch_inner=2))]
    bf = [t.to(torch.bfloat16) for t in (x, w)]
    good.append(tuple((t, qmm.operand(t, qmm.BF16, is_codes=False)) for t in bf))
    raw = qmm.operand(x, qmm.E4M3, torch.ones(1))
    good.append(((x, qmm.Operand(raw.data, raw.format, 1, raw.delta, raw.gran)), whole[1]))           # a descriptor of the caller's own
    for a, b in good:
        with pytest.raises(Reached):
            qmm.gemm_gated(a, b)
    bad = [(op(x, 3, per_channel=True), whole[1]), (whole[0], op(w, 10, per_channel=True)),             # the gate's step sizes only
           (op(codes(6, 4, 32), 2 * 4, per_channel=True, batch_groups=3), op(codes(6, 20, 32), 1)),
           (whole[0], (codes(22, 32), whole[1][1])), (op(codes(4, 16), 4, per_channel=True), (w[:, :16], whole[1][1])),     # the descriptor of another tensor
           ((x, qmm.operand(x, qmm.E4M3, torch.ones(4, dtype=torch.float64))), whole[1]),
           ((x, qmm.operand(x, qmm.E4M3, torch.ones(8)[::2], per_channel=True)), whole[1]),
           tuple((t, qmm.operand(t, qmm.BF16, is_codes=False)) for t in (x, w)),                        # bytes as bfloat16
           ((bf[0], qmm.operand(bf[0], qmm.E4M3, torch.ones(1))), whole[1])]
    for a, b in bad:
        with pytest.raises(ValueError):
            qmm.gemm_gated(a, b)
