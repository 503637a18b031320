"""The operators with a step size for every block of 128, layer norm and dropout on the CPU: their references against differences and known answers, and
the refusals of the C entries and of the binding, all of them made before anything is launched."""
import ctypes
import os

import numpy as np
import pytest
import torch

import block_reference as B
from paper_2408_02897_amd import qmm

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
OK, NULL, SHAPE, ENUM, ALIGN, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(qmm.LIB_PATH):
        from paper_2408_02897_amd import build
        build.build()
    return qmm.lib()


def T(rows=4, cols=256, dtype=qmm.DT_BF16, axis=1, batch=1, row_stride=None, batch_stride=None, data=FAKE):
    row_stride = cols if row_stride is None else row_stride
    return qmm.Tensor(data, dtype, axis, batch, rows, cols, rows * row_stride if batch_stride is None else batch_stride, row_stride)


def R(t):
    return None if t is None else ctypes.byref(t)


# ------------------------------------------------------------------------------------------------ references
def test_generator_known_answers():
    # the published vectors of Philox4x32-10, as in golden/philox4x32_10_kat.txt
    path = os.path.join(os.path.dirname(__file__), "golden", "philox4x32_10_kat.txt")
    rows = [[int(w, 16) for w in line.split()] for line in open(path) if line.strip() and not line.startswith("#")]
    assert rows
    for row in rows:
        c, k, want = row[:4], row[4:6], row[6:10]
        got = B._philox(*(np.array([v], dtype=np.uint64) for v in c), *k)
        assert [int(g[0]) for g in got] == want


def test_dropped_share_and_pieces():
    keep, scale = B.kept((200000,), 0.1, 2 ** 63 + 11, 12345)
    q = 6554 / 65536
    assert abs(1 - keep.double().mean() - q) < 4.5 * (q * (1 - q) / 200000) ** 0.5 and abs(scale.item() * (1 - q) - 1) < 1e-7
    part, _ = B.kept((1001,), 0.1, 2 ** 63 + 11, 12345 + 777)
    assert torch.equal(part, keep[777:1778])


def test_layer_norm_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    h, w, b, dy, dr = n(3, 50), 1 + 0.3 * n(50), n(50), n(3, 50), n(3, 50)
    loss = lambda h, w, b: (B.norm(h, w, b, 1e-3)[0] * dy).sum() + (h * dr).sum()
    _, mean, rstd, _ = B.norm(h, w, b, 1e-3)
    dh, dw, db, *_ = B.norm_grad(dy, h, mean, rstd, w, dr)
    for value, grad, at in ((h, dh, 0), (w, dw, 1), (b, db, 2)):
        v, step = n(*value.shape), 1e-5
        args = [h, w, b]
        ends = []
        for s in (step, -step):
            args[at] = value + s * v
            ends.append(loss(*args))
        assert abs((ends[0] - ends[1]) / (2 * step) - (grad * v).sum()) < 1e-6


# ------------------------------------------------------------------------------------------------ refusals
def test_block_scale_counts(L):
    assert L.qmm_num_block_scales(2, 300, 1000, 1) == 2 * 8 * 300 and L.qmm_num_block_scales(2, 300, 1000, 128) == 2 * 8 * 3
    assert L.qmm_num_block_scales(0, 3, 3, 1) == 0 and L.qmm_num_block_scales(1, 3, 0, 1) == 0
    for bad in ((-1, 3, 3, 1), (1, -3, 3, 1), (1, 3, -3, 1), (1, 3, 3, 64), (1, 3, 3, 0)):
        assert L.qmm_num_block_scales(*bad) == -1


def test_quantize_blocks_refuses(L):
    def call(x=T(), fmt=qmm.E4M3, per=1, mode=0, d=FAKE, c=FAKE, dt=None, ct=None):
        return L.qmm_quantize_blocks(R(x), fmt, per, mode, 0, 0, d, c, dt, ct, None)
    assert call(x=None) == NULL and call(d=None) == NULL and call(c=None) == NULL and call(x=T(data=None)) == NULL
    assert call(dt=FAKE) == NULL and call(ct=FAKE) == NULL
    assert call(fmt=qmm.INT8) == UNSUPPORTED and call(fmt=3) == ENUM and call(per=64) == ENUM and call(per=0) == ENUM and call(mode=2) == ENUM
    assert call(x=T(dtype=2)) == ENUM and call(x=T(axis=2)) == ENUM
    assert call(x=T(rows=-1)) == SHAPE and call(x=T(row_stride=255)) == SHAPE and call(x=T(batch=2, batch_stride=1000)) == SHAPE
    assert call(x=T(batch=65536)) == UNSUPPORTED
    assert call(x=T(data=ODD)) == ALIGN and call(d=ODD) == ALIGN and call(dt=ODD, ct=FAKE) == ALIGN
    for empty in (T(rows=0), T(cols=0), T(batch=0)):
        assert call(x=empty, d=None, c=None) == OK


def test_gemm_blocks_refuses(L):
    op = lambda data=FAKE, fmt=qmm.E4M3, per=1, delta=FAKE: qmm.BlockOperand(data, fmt, per, delta)

    def call(a=op(), b=op(per=128), shape=(1, 16, 16, 32), y=FAKE, dtype=qmm.DT_BF16, ws=None, n=0):
        return L.qmm_gemm_blocks(R(a), R(b), *shape, y, dtype, ws, n, None)
    assert call(a=None) == NULL and call(b=None) == NULL and call(y=None) == NULL
    for bad in (op(data=None), op(delta=None)):
        assert call(a=bad) == NULL and call(b=bad) == NULL
    assert call(a=op(fmt=qmm.INT8)) == UNSUPPORTED and call(b=op(fmt=qmm.BF16)) == UNSUPPORTED and call(a=op(fmt=9)) == ENUM and call(b=op(per=2)) == ENUM
    assert call(dtype=2) == ENUM and call(shape=(-1, 16, 16, 32)) == SHAPE and call(shape=(1, 16, -1, 32)) == SHAPE
    assert call(shape=(1, 16, 16, 24)) == ALIGN and call(a=op(data=ctypes.c_void_p(0x1008))) == ALIGN and call(y=ctypes.c_void_p(0x1004)) == ALIGN
    assert call(b=op(delta=ctypes.c_void_p(0x1002))) == ALIGN
    assert call(shape=(1, 16, 16, (1 << 22) + 16)) == UNSUPPORTED and call(shape=(1, 1 << 31, 16, 32)) == UNSUPPORTED
    for empty in ((0, 16, 16, 32), (1, 0, 16, 32), (1, 16, 0, 32)):
        assert call(shape=empty, y=None) == OK
    assert L.qmm_gemm_blocks_workspace_size(1, 4096, 4096, 8192) == 0 and L.qmm_gemm_blocks_workspace_size(1, 0, 5, 128) == 0
    need = L.qmm_gemm_blocks_workspace_size(1, 256, 256, 8192)
    assert need >= 2 * 256 * 256 * 4 and need % (256 * 256 * 4) == 0
    big = (1, 256, 256, 8192)
    assert call(shape=big) == WORKSPACE and call(shape=big, ws=FAKE, n=need - 1) == WORKSPACE and call(shape=big, ws=ctypes.c_void_p(0x1008), n=need) == ALIGN


def test_dropout_refuses(L):
    call = lambda x=T(), p=0.1, out=FAKE: L.qmm_dropout(R(x), p, 0, 0, out, None)
    assert call(x=None) == NULL and call(out=None) == NULL and call(x=T(data=None)) == NULL
    for p in (-0.1, 1.5, float("nan"), float("inf")):
        assert call(p=p) == SHAPE
    assert call(x=T(dtype=3)) == ENUM and call(x=T(axis=5)) == ENUM and call(x=T(cols=-1)) == SHAPE and call(x=T(row_stride=10)) == SHAPE
    assert call(x=T(data=ODD)) == ALIGN and call(out=ODD) == ALIGN
    assert call(x=T(row_stride=300), out=FAKE) == SHAPE                       # over an input whose rows lie apart
    assert call(x=T(rows=0), out=None) == OK


def test_layernorm_refuses(L):
    def call(x=T(), r=None, w=None, b=None, wt=qmm.DT_F32, eps=1e-5, p=0.0, fmt=qmm.E4M3, block=128, mode=0, h=None, y=None, mean=None, rstd=None, d=FAKE, c=FAKE):
        return L.qmm_layernorm_quantize(R(x), R(r), w, b, wt, eps, p, 0, 0, fmt, block, mode, 0, 0, h, y, mean, rstd, d, c, None)
    other = ctypes.c_void_p(0x100000)
    assert call(x=None) == NULL and call(d=None) == NULL and call(c=None) == NULL and call(x=T(data=None)) == NULL
    assert call(r=T()) == NULL and call(p=0.1) == NULL                        # h has nowhere to go
    assert call(d=None, c=None) == NULL                                      # nothing is asked for
    assert call(fmt=3) == ENUM and call(fmt=-1) == ENUM and call(block=64) == ENUM and call(mode=3) == ENUM and call(wt=7) == ENUM and call(x=T(dtype=4)) == ENUM
    assert call(x=T(axis=0)) == UNSUPPORTED and call(x=T(cols=(1 << 22) + 1)) == UNSUPPORTED and call(x=T(batch=65536)) == UNSUPPORTED
    assert call(r=T(rows=5), h=other) == SHAPE and call(r=T(dtype=qmm.DT_F32), h=other) == UNSUPPORTED
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(eps=eps) == SHAPE
    for p in (-0.5, 2.0, float("nan")):
        assert call(p=p, h=other) == SHAPE
    assert call(x=T(row_stride=300), p=0.1, h=FAKE) == SHAPE and call(x=T(row_stride=300), y=FAKE) == SHAPE and call(p=0.1, h=other, y=other) == SHAPE
    assert call(x=T(data=ODD)) == ALIGN and call(y=ODD) == ALIGN and call(w=ODD) == ALIGN and call(b=ODD) == ALIGN and call(mean=ODD) == ALIGN and call(rstd=ODD) == ALIGN
    assert call(x=T(rows=0), d=None, c=None) == OK


def test_layernorm_backward_refuses(L):
    t = T()
    need = L.qmm_layernorm_backward_workspace_size(R(t))
    other, third = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x200000)

    def call(dy=t, h=T(data=other), mean=FAKE, rstd=FAKE, w=None, wt=qmm.DT_F32, r=None, p=0.0, dh=third, dx=None, dw=None, db=None, ws=FAKE, n=1 << 30):
        return L.qmm_layernorm_backward(R(dy), R(h), mean, rstd, w, wt, R(r), p, 0, 0, dh, dx, dw, db, ws, n, None)
    assert call(dy=None) == NULL and call(h=None) == NULL and call(mean=None) == NULL and call(rstd=None) == NULL and call(dh=None) == NULL
    assert call(p=0.1) == NULL and call(dw=FAKE) == NULL and call(db=FAKE) == NULL and call(p=1.1, dx=other) == SHAPE
    assert call(h=T(rows=5)) == SHAPE and call(h=T(dtype=qmm.DT_F32)) == UNSUPPORTED and call(r=T(cols=255)) == SHAPE and call(wt=9) == ENUM
    assert call(dy=T(row_stride=300), dh=FAKE) == SHAPE and call(p=0.1, dx=third) == SHAPE
    assert call(dh=ODD) == ALIGN and call(mean=ODD) == ALIGN and call(rstd=ODD) == ALIGN and call(w=ODD) == ALIGN and call(dw=ODD, db=FAKE) == ALIGN
    if need:
        assert call(dw=FAKE, db=FAKE, ws=None, n=0) == WORKSPACE and call(dw=FAKE, db=FAKE, n=need - 1) == WORKSPACE
        assert call(dw=FAKE, db=FAKE, ws=ctypes.c_void_p(0x1008)) == ALIGN
    assert L.qmm_layernorm_backward_workspace_size(R(T(rows=100000, cols=64))) > 0 and L.qmm_layernorm_backward_workspace_size(R(T(rows=0))) == 0


def test_binding_refuses():
    codes, delta = torch.zeros((4, 256), dtype=torch.uint8), torch.ones(2 * 4)
    qmm.block_operand(codes, qmm.E4M3, delta)
    for bad in (lambda: qmm.block_operand(codes.float(), qmm.E4M3, delta), lambda: qmm.block_operand(codes[:, :100], qmm.E4M3, delta),
                lambda: qmm.block_operand(codes, qmm.E4M3, delta[:7]), lambda: qmm.block_operand(codes, qmm.E4M3, delta.double()),
                lambda: qmm.block_operand(codes, qmm.E4M3, delta, block_rows=64), lambda: qmm.block_operand(codes, qmm.E4M3, delta, block_rows=128)):
        with pytest.raises(ValueError):
            bad()
    op = qmm.block_operand(codes, qmm.E4M3, delta)
    x = torch.zeros((4, 256))
    # host tensors: no kernel of this library may see them
    for bad in (lambda: qmm.gemm_blocks((codes, op), (codes, op)), lambda: qmm.quantize_blocks(x, 1, qmm.E4M3), lambda: qmm.dropout(x, 0.1, 0),
                lambda: qmm.layernorm_quantize(x, None, None), lambda: qmm.layernorm_backward(x, x, torch.zeros(4), torch.ones(4), None)):
        with pytest.raises(ValueError):
            bad()


def test_step_sizes_in_another_order_are_refused():
    """As many step sizes as the operand has, laid out [rows, blocks] or for other matrices: another matrix's, by the product's rule."""
    for codes, per, good, bad in ((torch.zeros((256, 256), dtype=torch.uint8), 1, ((512,), (2, 256), (1, 2, 256)), ((256, 2), (1, 256, 2), (2, 256, 1), (2, 1, 256), (1, 1, 2, 256))),
                                  (torch.zeros((300, 1024), dtype=torch.uint8), 128, ((24,), (8, 3), (1, 8, 3)), ((3, 8), (1, 3, 8), (8, 3, 1))),
                                  (torch.zeros((2, 40, 272), dtype=torch.uint8), 1, ((240,), (2, 3, 40)), ((2, 40, 3), (3, 80), (6, 40), (3, 2, 40), (3, 40, 2))),
                                  (torch.zeros((1, 40, 272), dtype=torch.uint8), 1, ((120,), (3, 40), (1, 3, 40)), ((40, 3), (1, 40, 3)))):
        for shape in good:
            qmm.block_operand(codes, qmm.E4M3, torch.ones(shape), block_rows=per)
        for shape in bad:
            with pytest.raises(ValueError, match="step sizes"):
                qmm.block_operand(codes, qmm.E4M3, torch.ones(shape), block_rows=per)


def test_operands_changed_since_they_were_made_are_refused():
    """With block_rows set to 1 where there are step sizes per 128 rows the product would read past them."""
    codes, other = torch.zeros((300, 256), dtype=torch.uint8), torch.zeros((300, 256), dtype=torch.uint8)
    make = lambda per: qmm.block_operand(codes, qmm.E4M3, torch.ones((2, -(-300 // per))), block_rows=per)
    for per in (1, 128):
        qmm._check_block_operand(codes, make(per))
        op = make(per)
        op.block_rows = 129 - per
        with pytest.raises(ValueError, match="step sizes"):
            qmm._check_block_operand(codes, op)
        with pytest.raises(ValueError, match="another tensor"):
            qmm._check_block_operand(other, make(per))
    with pytest.raises(ValueError, match="block_operand"):
        qmm._check_block_operand(codes, qmm.BlockOperand(codes.data_ptr(), qmm.E4M3, 1, 0))


def test_quantize_blocks_extents(L):
    """Up to 2^31 - 129 elements along either axis, as the header says (refused before the step sizes' missing place is)."""
    call = lambda x: L.qmm_quantize_blocks(R(x), qmm.E4M3, 1, 0, 0, 0, None, None, None, None, None)
    most = 2 ** 31 - 129
    for axis in (0, 1):
        assert call(T(rows=most, cols=1, axis=axis)) == NULL and call(T(rows=1, cols=most, axis=axis)) == NULL
        assert call(T(rows=most + 1, cols=1, axis=axis)) == UNSUPPORTED and call(T(rows=1, cols=most + 1, axis=axis)) == UNSUPPORTED
