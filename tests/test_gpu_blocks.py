"""Step sizes per block of 128 on the GPU: codes bit for bit against qmm_scale_quantize and qmm_quantize of the blocks alone, products against binary64
(tests/block_reference.py); dropout bit for bit against its generator written down in numpy."""
import pytest
import torch

import block_forms as F
import block_reference as B
import ffn_reference as R
from paper_2408_02897_amd import qmm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
FORMATS = [qmm.E4M3, qmm.E5M2]


def normal(seed, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def apart(t, rows=2, cols=3):
    """The same values with `rows` rows between the matrices and `cols` elements between the rows, off a 16-byte boundary, NaN in between."""
    t3 = t if t.dim() == 3 else t.unsqueeze(0)
    b, r, c = t3.shape
    big = torch.full((b * (r + rows) * (c + cols) + 1,), float("nan"), dtype=t.dtype, device=DEV)[1:].view(b, r + rows, c + cols)
    v = big[:, :r, :c]
    v.copy_(t3)
    return v if t.dim() == 3 else v[0]


# ------------------------------------------------------------------------------------------------ codes
def blocks_alone(x, fmt, per, mode=qmm.RTNE, seed=0, offset=0):
    """codes and delta of x [batch, rows, k] (on the GPU), every block through the calls for whole tensors."""
    b, r, k = x.shape
    codes = torch.empty((b, r, k), dtype=torch.uint8, device=DEV)
    delta = torch.empty((b, -(-k // 128), -(-r // per)), device=DEV)
    for i in range(b):
        for kb in range(delta.shape[1]):
            ks = slice(128 * kb, min(128 * kb + 128, k))
            if per == 1 and mode == qmm.RTNE:
                codes[i, :, ks], delta[i, kb] = (t[0] if t.dim() == 3 else t for t in qmm.scale_quantize(x[i, :, ks].contiguous(), 1, fmt, per_channel=True))
                continue
            for rb in range(delta.shape[2]):
                rs = slice(per * rb, min(per * rb + per, r))
                part = x[i, rs, ks].contiguous()
                delta[i, kb, rb] = qmm.scale(part, 1, fmt)[0]
                for row in range(rs.start, rs.stop):           # (a row at a time: its codes' places are side by side)
                    codes[i, row:row + 1, ks] = qmm.quantize(x[i, row:row + 1, ks].contiguous(), 1, fmt, delta[i, kb, rb:rb + 1].contiguous(), mode=mode, seed=seed,
                                                             offset=offset + (i * r + row) * k + ks.start)[0]
    return codes, delta


SIZES = [(1, 1), (1, 4096), (3, 7), (5, 128), (17, 129), (33, 100), (128, 128), (127, 255), (130, 400), (260, 1000), (1, 5000), (300, 17)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_codes_by_rows(rows, cols, dtype):
    x = normal(rows + cols, rows, cols, scale=3.0)
    x[0, 0] = 0.0 if rows * cols > 1 else 1.0
    x = x.to(dtype).to(DEV)
    for fmt in FORMATS:
        want = blocks_alone(x.unsqueeze(0), fmt, 1), blocks_alone(x.t().contiguous().unsqueeze(0), fmt, 1)
        for v in (x, apart(x)):
            (c, d), (ct, dt) = qmm.quantize_blocks(v, 1, fmt, both=True)
            for got, w in ((c, want[0][0]), (d, want[0][1]), (ct, want[1][0]), (dt, want[1][1])):
                assert R.same_bits(got, w)
            for axis in (1, 0):
                got = qmm.quantize_blocks(v, axis, fmt)
                assert R.same_bits(got[0], want[1 - axis][0]) and R.same_bits(got[1], want[1 - axis][1])
            (ct, dt), (c, d) = qmm.quantize_blocks(v, 0, fmt, both=True)
            assert R.same_bits(c, want[0][0]) and R.same_bits(dt, want[1][1])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 300), (5, 128), (127, 255), (128, 128), (130, 260)])
def test_codes_by_squares(rows, cols, dtype):
    x = normal(rows + cols, rows, cols, dtype=dtype, scale=0.02).to(DEV)
    for fmt in FORMATS:
        want = blocks_alone(x.unsqueeze(0), fmt, 128)
        for v in (x, apart(x)):
            (c, d), (ct, dt) = qmm.quantize_blocks(v, 1, fmt, block_rows=128, both=True)
            assert R.same_bits(c, want[0]) and R.same_bits(d, want[1])
            assert R.same_bits(ct, want[0].transpose(1, 2).contiguous()) and R.same_bits(dt, want[1].transpose(1, 2).contiguous())
            for axis in (0, 1):
                got = qmm.quantize_blocks(v, axis, fmt, block_rows=128)
                assert R.same_bits(got[0], c if axis else ct) and R.same_bits(got[1], d if axis else dt)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("rows,cols,offset", [(9, 200, 0), (6, 135, 7), (130, 20, 2)])
def test_codes_batches_and_stochastic_rounding(rows, cols, offset, per, dtype):
    x = normal(1, 2, rows, cols, dtype=dtype).to(DEV)
    for fmt in FORMATS:
        kw = dict(mode=qmm.STOCHASTIC, seed=2 ** 63 + 7, offset=offset)
        want = blocks_alone(x, fmt, per, **kw), blocks_alone(x.transpose(1, 2).contiguous(), fmt, per, **kw)
        for v in (x, apart(x)):
            (c, d), (ct, dt) = qmm.quantize_blocks(v, 1, fmt, block_rows=per, both=True, **kw)
            assert R.same_bits(c, want[0][0]) and R.same_bits(d, want[0][1]) and R.same_bits(ct, want[1][0]) and R.same_bits(dt, want[1][1])
            for axis in (0, 1):
                got = qmm.quantize_blocks(v, axis, fmt, block_rows=per, **kw)
                assert R.same_bits(got[0], want[1 - axis][0]) and R.same_bits(got[1], want[1 - axis][1])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_codes_of_special_values(dtype):
    x = normal(1, 140, 300)
    x[1] = 0.0
    x[2, 3], x[3, 130], x[4, 299] = float("inf"), float("nan"), float("-inf")
    x[5] = 1e-38
    x[6] = 3e38
    x[7] = -0.0
    x = x.to(dtype).to(DEV)
    for fmt in FORMATS:
        for per in (1, 128):
            (c, d), (ct, dt) = qmm.quantize_blocks(x, 1, fmt, block_rows=per, both=True)
            w, wt = blocks_alone(x.unsqueeze(0), fmt, per), blocks_alone(x.t().contiguous().unsqueeze(0), fmt, per)
            for got, want in ((c, w[0]), (ct, wt[0])):
                assert torch.equal(got, want)
            for got, want in ((d, w[1]), (dt, wt[1])):
                assert torch.equal(torch.nan_to_num(got, nan=-1.0), torch.nan_to_num(want, nan=-1.0))
    for shape in ((0, 5), (5, 0), (2, 0, 3)):
        c, d = qmm.quantize_blocks(torch.empty(shape, dtype=dtype, device=DEV), 1, qmm.E4M3)
        assert c.numel() == 0 and d.numel() == 0


def test_codes_of_a_large_tensor():
    """More rows than a grid dimension takes, offsets past 32 bits in the codes' places of the transposed tensor."""
    x = torch.randn((70000, 136), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV, dtype=BF)
    (c, d), (ct, dt) = qmm.quantize_blocks(x, 1, qmm.E5M2, both=True)
    w, wd = qmm.scale_quantize(x[:, :128].contiguous(), 1, qmm.E5M2, per_channel=True)
    assert torch.equal(c[0, :, :128], w[0]) and torch.equal(d[0, 0], wd)
    last = x[69888:].t().contiguous()
    w, wd = qmm.scale_quantize(last, 1, qmm.E5M2, per_channel=True)
    assert torch.equal(ct[0, :, 69888:], w[0]) and torch.equal(dt[0, -1], wd)


@pytest.mark.parametrize("mode", [qmm.RTNE, qmm.STOCHASTIC])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_codes_of_many_rows_are_those_of_their_pieces(dtype, mode):
    """Enough rows for tiles, along one axis alone; NaN and infinities in some blocks, the others of their tiles untouched."""
    rows, cols = 40077, 200
    x = torch.randn((rows, cols), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(dtype)
    for at, v in (((5, 7), float("nan")), ((200, 199), float("inf")), ((201, 3), -float("inf")), ((40076, 150), float("nan"))):
        x[at] = v
    x[300] = 0
    for v in (x, apart(x.cpu())):
        for per in (1, 128):
            c, d = qmm.quantize_blocks(v, 1, qmm.E4M3, block_rows=per, mode=mode, seed=3, offset=6)
            for first, last in ((0, 384), (19968, 20480), (39936, rows)):
                pc, pd = qmm.quantize_blocks(x[first:last], 1, qmm.E4M3, block_rows=per, mode=mode, seed=3, offset=6 + first * cols)
                assert torch.equal(c[:, first:last], pc)
                assert torch.equal(torch.nan_to_num(d[..., first // per:-(-last // per)], nan=-1.0), torch.nan_to_num(pd, nan=-1.0))


def test_elements_past_32_bits():
    """2^31 and more elements of each operator: their last rows are what the operator makes of these alone."""
    before, rest, cols = 2 ** 19, 300, 4096
    x = torch.empty((before + rest, cols), device=DEV, dtype=BF)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(4))
    tail = x[before:].clone()
    (c, d), (ct, dt) = qmm.quantize_blocks(x, 1, qmm.E4M3, both=True)
    (pc, pd), (pct, pdt) = qmm.quantize_blocks(tail, 1, qmm.E4M3, both=True)
    assert torch.equal(c[:, before:], pc) and torch.equal(d[..., before:], pd)
    assert torch.equal(ct[..., before:], pct) and torch.equal(dt[:, before // 128:], pdt)
    del ct, dt, pct, pdt
    w = normal(5, 1, 4096, 256, scale=0.05).to(DEV)
    cw, dw = qmm.quantize_blocks(w, 1, qmm.E4M3, block_rows=128)
    b = cw, qmm.block_operand(cw, qmm.E4M3, dw, block_rows=128)
    k, kd = c[..., :256].contiguous(), d[:, :2].contiguous()
    y = qmm.gemm_blocks((k, qmm.block_operand(k, qmm.E4M3, kd)), b, BF)
    pk, pkd = k[:, before:].contiguous(), kd[..., before:].contiguous()
    assert R.same_bits(y[:, before:], qmm.gemm_blocks((pk, qmm.block_operand(pk, qmm.E4M3, pkd)), b, BF))     # (two blocks: no split)
    del c, d, k, kd
    assert R.same_bits(qmm.dropout(x, 0.1, 5, 3, out=y[0])[before:], qmm.dropout(tail, 0.1, 5, 3 + before * cols))
    weight, bias = normal(6, cols).to(DEV).to(BF), normal(7, cols).to(DEV).to(BF)
    dropping = dict(dropout=0.1, dropout_seed=8)
    n = qmm.layernorm_quantize(x, weight, bias, fmt=qmm.E4M3, block=True, residual=x, want_y=True, want_stats=True, dropout_offset=1, **dropping)
    p = qmm.layernorm_quantize(tail, weight, bias, fmt=qmm.E4M3, block=True, residual=tail, want_y=True, want_stats=True, dropout_offset=1 + before * cols, **dropping)
    assert torch.equal(n.codes[:, before:], p.codes) and torch.equal(n.delta[..., before:], p.delta)
    for name in ("h", "y"):
        assert R.same_bits(getattr(n, name).reshape(-1, cols)[before:], getattr(p, name).reshape(-1, cols))
    mean, rstd = n.mean.reshape(-1), n.rstd.reshape(-1)
    assert torch.equal(mean[before:], p.mean.reshape(-1)) and torch.equal(rstd[before:], p.rstd.reshape(-1))
    h = n.h.reshape(-1, cols)
    g = qmm.layernorm_backward(x, h, mean, rstd, weight, dresidual=x, want_dw=False, dropout_offset=1, **dropping)
    q = qmm.layernorm_backward(tail, h[before:].clone(), mean[before:].clone(), rstd[before:].clone(), weight, dresidual=tail, want_dw=False,
                               dropout_offset=1 + before * cols, **dropping)
    assert R.same_bits(g.dh.reshape(-1, cols)[before:], q.dh.reshape(-1, cols)) and R.same_bits(g.dx.reshape(-1, cols)[before:], q.dx.reshape(-1, cols))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_codes_of_more_tiles_than_a_launch_takes(dtype):
    """65535 matrices of one row: 65 tiles each, in all more than 2^32 threads' worth in binary32.  Row by row they are those of one matrix with as many rows."""
    x = torch.randn((65535, 1, 8320), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV, dtype=dtype)
    want, step = qmm.quantize_blocks(x[:, 0], 1, qmm.E4M3)
    (c, d), (ct, dt) = qmm.quantize_blocks(x, 1, qmm.E4M3, both=True)
    assert torch.equal(c[:, 0], want[0]) and torch.equal(d[:, :, 0], step[0].t())
    for first, last in ((0, 3), (32767, 32771), (65532, 65535)):
        pt, pdt = qmm.quantize_blocks(x[first:last], 0, qmm.E4M3)
        assert torch.equal(ct[first:last], pt) and torch.equal(dt[first:last], pdt)


# ------------------------------------------------------------------------------------------------ product
def operands(seed, batch, m, n, k, fa, fb, per_a, per_b):
    x, w = normal(seed, batch, m, k, scale=2.0).to(DEV), normal(seed + 1, batch, n, k, scale=0.05).to(DEV)
    (ca, da), (cb, db) = qmm.quantize_blocks(x, 1, fa, block_rows=per_a), qmm.quantize_blocks(w, 1, fb, block_rows=per_b)
    return (ca, qmm.block_operand(ca, fa, da, block_rows=per_a)), (cb, qmm.block_operand(cb, fb, db, block_rows=per_b)), (ca, cb, da, db, fa, fb, per_a, per_b)


def check_product(a, b, what):
    y, off = B.product(*what)
    for dtype in (F32, BF):
        got = qmm.gemm_blocks(a, b, dtype)
        assert got.shape == y.shape and got.dtype == dtype
        bound = off + R.rounding(dtype) * (y.abs() + off) if dtype == BF else off
        d = (got.double() - y).abs()
        assert torch.all(d <= bound), ((d - bound).max().item(), d.max().item())
        assert R.same_bits(got, qmm.gemm_blocks(a, b, dtype))


PRODUCTS = [(1, 1, 16), (1, 33, 64), (2, 100, 4096), (1, 512, 2048), (5, 64, 272), (16, 256, 1024), (17, 130, 144), (33, 96, 400), (64, 64, 128), (65, 63, 128),
            (100, 200, 304), (129, 129, 144), (130, 257, 1040), (256, 128, 512), (300, 640, 384), (512, 256, 256), (1031, 100, 784), (1024, 1024, 96), (3, 1000, 6160),
            (70, 61, 4096), (200, 130, 2064), (129, 512, 4080), (257, 257, 2192), (400, 1, 160), (2000, 2100, 400)]


@pytest.mark.parametrize("fa,fb", [(qmm.E4M3, qmm.E4M3), (qmm.E4M3, qmm.E5M2), (qmm.E5M2, qmm.E4M3), (qmm.E5M2, qmm.E5M2)])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, fa, fb):
    for per_a, per_b in ((1, 128), (1, 1)) if (fa, fb) != (qmm.E4M3, qmm.E4M3) else ((1, 128), (1, 1), (128, 128), (128, 1)):
        check_product(*operands(m + n + k, 1, m, n, k, fa, fb, per_a, per_b))


@pytest.mark.parametrize("batch,m,n,k", [(3, 1, 40, 96), (5, 20, 64, 128), (2, 150, 130, 272), (3, 300, 200, 128), (3, 7, 50, 6400), (2, 130, 70, 4096), (40, 260, 300, 144)])
def test_product_in_batches(batch, m, n, k):
    for per_a, per_b in ((1, 128), (1, 1), (128, 128)):
        check_product(*operands(k, batch, m, n, k, qmm.E4M3, qmm.E4M3, per_a, per_b))


@pytest.mark.parametrize("m,n,k", [(4096, 3328, 512), (3585, 4097, 400), (8200, 1800, 1168)])
def test_product_of_many_tiles(m, n, k):
    for per_a, per_b in ((1, 128), (1, 1)):
        check_product(*operands(k, 1, m, n, k, qmm.E5M2, qmm.E4M3, per_a, per_b))


@pytest.mark.parametrize("batch,m,n,k,tile,splits,groups", F.FORMS)
def test_product_by_every_form(batch, m, n, k, tile, splits, groups):
    """Step sizes per row and per 128 rows of either operand, both output types; what lies around the output stays as it was."""
    for fa, fb, per_a, per_b in ((qmm.E4M3, qmm.E4M3, 1, 128), (qmm.E5M2, qmm.E4M3, 1, 1), (qmm.E4M3, qmm.E5M2, 128, 128)):
        a, b, what = operands(m + n + k, batch, m, n, k, fa, fb, per_a, per_b)
        check_product(a, b, what)
        for dtype in (F32, BF):
            room = torch.full((batch * m * n + 4096,), 7.0, dtype=dtype, device=DEV)
            out = room[2048:-2048].view(batch, m, n)
            qmm.gemm_blocks(a, b, out=out)
            assert torch.all(room[:2048] == 7) and torch.all(room[-2048:] == 7) and torch.equal(out, qmm.gemm_blocks(a, b, dtype))


@pytest.mark.parametrize("batch,m,n,k,tile,splits,groups", F.LARGE[:3] + F.LARGE_SPLIT[1:4] + F.MIDDLE[:2] + F.MIDDLE_SPLIT[3:5] + F.SMALL[1:2] + F.FEW[1:3])
def test_not_a_number_in_one_row(batch, m, n, k, tile, splits, groups):
    """Codes and step sizes that are not finite reach their rows' and columns' outputs and no others, those of a workgroup's next tile among them."""
    for per_b in (1, 128):
        a, b, what = operands(5, batch, m, n, k, qmm.E4M3, qmm.E4M3, 1, per_b)
        want = qmm.gemm_blocks(a, b, F32)
        ca, cb, da, db = (t.clone() for t in what[:4])
        i, j, z = m // 2, n - 1, batch - 1
        ca[z, i, k - 1] = 0x7F
        cb[z, j, 0] = 0x7F
        da[z, -1, 0] = float("nan")
        got = qmm.gemm_blocks((ca, qmm.block_operand(ca, qmm.E4M3, da)), (cb, qmm.block_operand(cb, qmm.E4M3, db, block_rows=per_b)), F32)
        hit = torch.zeros((batch, m, n), dtype=torch.bool, device=DEV)
        hit[z, i], hit[z, :, j], hit[z, 0] = True, True, True
        assert torch.equal(torch.isnan(got), hit) and torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("m,n", [(1, 64), (40, 70), (100, 200), (300, 130), (4096, 3200)])
def test_a_block_is_the_plain_products_sum(m, n):
    """One block and step sizes of one: the accumulators of qmm_gemm, bit for bit."""
    x, w = normal(1, 1, m, 128, scale=50.0).to(DEV), normal(2, 1, n, 128, scale=50.0).to(DEV)
    one = torch.ones(max(m, n), device=DEV)
    a, b = qmm.quantize(x, 1, qmm.E4M3, one[:1]), qmm.quantize(w, 1, qmm.E4M3, one[:1])
    want = qmm.gemm((a, qmm.operand(a, qmm.E4M3, one)), (b, qmm.operand(b, qmm.E4M3, one)), F32)
    for per in (1, 128):
        oa, ob = (qmm.block_operand(c, qmm.E4M3, torch.ones(1, 1, -(-c.shape[1] // per), device=DEV), block_rows=per) for c in (a, b))
        assert R.same_bits(qmm.gemm_blocks((a, oa), (b, ob), F32), want)


@pytest.mark.parametrize("m", [1, 40, 100, 300])
def test_product_edges(m):
    """No contraction, no rows; a NaN and an infinity in one row of an operand or one step size touch that row's outputs only."""
    e = lambda r: torch.empty((r, 0), dtype=torch.uint8, device=DEV)
    none = torch.empty(0, device=DEV)
    y = qmm.gemm_blocks((e(m), qmm.block_operand(e(m), qmm.E4M3, none)), (e(80), qmm.block_operand(e(80), qmm.E4M3, none, block_rows=128)), F32)
    assert y.shape == (1, m, 80) and torch.all(y == 0)
    a, b, what = operands(1, 1, m, 150, 336, qmm.E4M3, qmm.E4M3, 1, 1)
    want = qmm.gemm_blocks(a, b, F32)
    ca, cb, da, db = (t.clone() for t in what[:4])
    cb[0, 20, 300] = 0x7F
    db[0, 1, 40] = float("inf")
    da[0, 2, m - 1] = float("nan")
    got = qmm.gemm_blocks((ca, qmm.block_operand(ca, qmm.E4M3, da)), (cb, qmm.block_operand(cb, qmm.E4M3, db)), F32)
    assert torch.isnan(got[0, :, 20]).all() and not torch.isfinite(got[0, :, 40]).any() and torch.isnan(got[0, m - 1]).all()
    rest = [i for i in range(150) if i not in (20, 40)]
    assert torch.equal(got[0, :m - 1, rest], want[0, :m - 1, rest])
    zero = torch.empty((0, 32), dtype=torch.uint8, device=DEV)
    assert qmm.gemm_blocks((zero, qmm.block_operand(zero, qmm.E4M3, none)), (zero, qmm.block_operand(zero, qmm.E4M3, none))).shape == (1, 0, 0)


def test_product_writes_its_rows_only():
    a, b, _ = operands(3, 1, 200, 136, 256, qmm.E4M3, qmm.E4M3, 1, 128)
    want = qmm.gemm_blocks(a, b, BF)
    big = torch.full((240, 136), 7.0, dtype=BF, device=DEV)
    out = big[16:216].view(1, 200, 136)
    assert qmm.gemm_blocks(a, b, out=out) is out and R.same_bits(out, want) and torch.all(big[:16] == 7) and torch.all(big[216:] == 7)


def test_operands_of_other_tensors():
    a, b, what = operands(3, 1, 20, 30, 256, qmm.E4M3, qmm.E4M3, 1, 128)
    for bad in (((a[0].clone(), a[1]), b), (a, (b[0][:, :20], b[1])), (a, (b[0].float(), b[1]))):
        with pytest.raises((ValueError, AssertionError)):
            qmm.gemm_blocks(*bad)


@pytest.mark.parametrize("short", [None, qmm._NoShortPath])
def test_operands_changed_since_they_were_made(short, monkeypatch):
    monkeypatch.setattr(qmm, "_short", short)
    for per_a, per_b in ((1, 128), (128, 1)):
        for which in range(2):
            pairs = operands(3, 1, 200, 300, 256, qmm.E4M3, qmm.E4M3, per_a, per_b)[:2]
            qmm.gemm_blocks(*pairs)
            pairs[which][1].block_rows = 129 - pairs[which][1].block_rows
            with pytest.raises(ValueError, match="step sizes"):
                qmm.gemm_blocks(*pairs)


@pytest.mark.parametrize("m,n,k", [(300, 1000, 8192), (100, 512, 4096), (4096, 3328, 256)])
def test_products_recorded_and_at_once(m, n, k):
    """Two graphs of the same product (parts of a contraction in a workspace of each one's own; workgroups that stay) replayed in turn and side by side, codes
    changing, an eager call between."""
    sets = [operands(7 * i + 1, 1, m, n, k, qmm.E4M3, qmm.E4M3, 1, 128) for i in range(3)]
    want = [qmm.gemm_blocks(a, b, BF) for a, b, _ in sets]
    runs = []
    for i in range(2):
        ca, cb, da, db = (t.clone() for t in sets[i][2][:4])
        a, b = (ca, qmm.block_operand(ca, qmm.E4M3, da)), (cb, qmm.block_operand(cb, qmm.E4M3, db, block_rows=128))
        qmm.gemm_blocks(a, b, BF)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = qmm.gemm_blocks(a, b, BF)
        runs.append((g, y, (ca, cb, da, db)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(3):
        for i, (g, y, parts) in enumerate(runs):
            for to, of in zip(parts, sets[(turn + i) % 3][2]):
                to.copy_(of)
        torch.cuda.synchronize()
        for s, (g, y, parts) in zip(streams, runs):
            with torch.cuda.stream(s):
                g.replay()
        assert R.same_bits(qmm.gemm_blocks(*sets[turn][:2], BF), want[turn])
        torch.cuda.synchronize()
        for i, (g, y, parts) in enumerate(runs):
            assert R.same_bits(y, want[(turn + i) % 3])


@pytest.mark.parametrize("batch,m,n,k,tile,splits,groups", [F.LARGE[0], F.LARGE_SPLIT[0], F.LARGE_SPLIT[2], F.MIDDLE_SPLIT[0], F.MIDDLE_SPLIT[1]])
def test_products_of_large_forms_recorded_and_at_once(batch, m, n, k, tile, splits, groups):
    """Workgroups that go from tile to tile, and parts of a contraction in 256 x 256 and 128 x 128, in two graphs side by side."""
    assert batch == 1
    test_products_recorded_and_at_once(m, n, k)


@pytest.mark.parametrize("batch,m", [(2 ** 24 - 1, 1), (2 ** 24 + 5, 2)])
def test_product_of_more_matrices_than_a_launch_takes(batch, m):
    """A workgroup a matrix, up to 2^32 threads and beyond."""
    g = torch.Generator(device=DEV).manual_seed(batch)
    code = lambda r: torch.randint(0, 0x78, (batch, r, 16), generator=g, device=DEV, dtype=torch.uint8)        # (finite and positive)
    ca, cb = code(m), code(1)
    da, db = (torch.rand((batch, 1, r), generator=g, device=DEV) + 0.5 for r in (m, 1))
    got = qmm.gemm_blocks((ca, qmm.block_operand(ca, qmm.E4M3, da)), (cb, qmm.block_operand(cb, qmm.E4M3, db)), F32)
    for i in range(m):
        va, vb = B.decode(ca[:, i], qmm.E4M3), B.decode(cb[:, 0], qmm.E4M3)
        step = da[:, 0, i].double() * db[:, 0, 0].double()
        y, cut = (va * vb).sum(1) * step, (B.power(va, qmm.E4M3) * B.power(vb, qmm.E4M3)).sum(1) * step
        assert torch.all((got[:, i, 0].double() - y).abs() <= 7.0 * 2.0 ** -13 * cut + 32 * R.EPS32 * y + 2.0 ** -120)      # (as in block_reference.product)


# ------------------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("shape", [(1, 1), (1, 4096), (3, 7), (67, 100), (2, 9, 129), (3, 50, 8)])
def test_dropout(shape, dtype):
    x = normal(3, *shape, dtype=dtype, scale=2.0)
    for p, seed, offset in ((0.1, 0, 0), (0.5, 2 ** 63 + 3, 5), (0.25, 2 ** 64 - 1, 2 ** 40 + 6), (0.9, 17, 2 ** 64 - 3)):
        want = B.dropped(x, p, seed, offset)
        assert R.same_bits(qmm.dropout(x.to(DEV), p, seed, offset), want)
        assert R.same_bits(qmm.dropout(apart(x), p, seed, offset), want)
        y = x.to(DEV)
        assert qmm.dropout(y, p, seed, offset, out=y) is y and R.same_bits(y, want)
    assert R.same_bits(qmm.dropout(x.to(DEV), 0.0, 1), x) and torch.all(qmm.dropout(x.to(DEV), 1.0, 1) == 0) and R.same_bits(qmm.dropout(x.to(DEV), 1e-6, 1), x)


def test_dropout_of_a_whole_and_its_parts():
    x = normal(1, 40000, 1000, dtype=BF).to(DEV)               # beyond 64 MB: past the caches
    y = qmm.dropout(x, 0.1, 5, 3)
    for first, last in ((0, 1), (777, 1781), (39990, 40000)):
        assert R.same_bits(y[first:last], qmm.dropout(x[first:last], 0.1, 5, 3 + first * 1000))
    special = torch.tensor([[float("nan"), float("inf"), -float("inf"), -0.0] * 64], device=DEV)
    keep, scale = B.kept(special.shape, 0.5, 9, 0)
    got = qmm.dropout(special, 0.5, 9).cpu()
    assert torch.all(got[~keep] == 0) and torch.isnan(got[keep][0::1][torch.isnan(special.cpu()[keep])]).all()
    assert qmm.dropout(torch.empty((0, 5), device=DEV), 0.1, 0).shape == (0, 5)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_dropout_numbers_start_again_behind_the_last(dtype):
    """Element numbers are modulo 2^64: within a vector that holds the last and the first of them too, for offsets given as negative numbers as well."""
    x = torch.ones((2, 40), dtype=dtype)
    for back in range(1, 18):
        for seed in range(4):
            want = B.dropped(x, 0.5, seed, 2 ** 64 - back)
            for offset in (2 ** 64 - back, -back):
                assert R.same_bits(qmm.dropout(x.to(DEV), 0.5, seed, offset), want)
            whole = qmm.dropout(torch.ones((1, 40 + back), dtype=dtype, device=DEV), 0.5, seed, -back)
            assert R.same_bits(whole[:, back:], qmm.dropout(torch.ones((1, 40), dtype=dtype, device=DEV), 0.5, seed, 0))
