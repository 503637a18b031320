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
