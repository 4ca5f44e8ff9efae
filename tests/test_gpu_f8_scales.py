"""Scales of the 8-bit float layer at both ends of their range: of any finite size where the product of a row's and a column's is a normal
number or 0, or the block's codes are zeros."""
import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests import f8_ref
from tests.test_gpu_f8_layer import F8, FMT, round16, stream

pytestmark = pytest.mark.gpu

# rows and filters of every form: split over 16, 32 and 64 rows, single tiles, pairs of tiles
FORMS = [(3, 200, 700), (16, 130, 1500), (30, 300, 260), (64, 200, 1300), (200, 300, 300), (2600, 2700, 260)]


def codes_of(values, fmt):
    ld = round16(values.shape[1])
    q = torch.full((values.shape[0], ld), 0x7F, dtype=torch.uint8, device="cuda")
    q[:, :values.shape[1]] = torch.from_numpy(values).to(torch.float32).to(F8[fmt]).view(torch.uint8).cuda()
    return q


def layer(xv, sx, wv, sw, w_block, xf, wf):
    """The call's y (fp32), and in 64 bits what it stands for, the sum of magnitudes, and that of its blocks' sums."""
    M, C = xv.shape
    K = wv.shape[0]
    x, w = codes_of(xv, xf), codes_of(wv, wf)
    dsx, dsw = torch.from_numpy(sx).cuda(), torch.from_numpy(sw).cuda()
    y = torch.full((M, K), -77.0, device="cuda")
    d = sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=K, Cmax=C, x_format=FMT[xf], w_format=FMT[wf], w_block_rows=w_block, y_dtype=sgs.SGS_F32)
    sgs.linear_f8(d, x.data_ptr(), dsx.data_ptr(), w.data_ptr(), dsw.data_ptr(), 0, y.data_ptr(), stream())
    torch.cuda.synchronize()
    assert sgs.device_status() == 0
    ref, size = f8_ref.linear(xv, sx, wv, sw, w_block, None, 0, M, K, C)
    reach = np.zeros((M, K))
    for b in range(sx.shape[0]):
        at = slice(128 * b, min(C, 128 * b + 128))
        reach += np.abs((xv[:, at] @ wv[:, at].T) * sx[b].astype(np.float64)[:, None] * sw[b].astype(np.float64)[np.arange(K) // w_block])
    return y.double().cpu().numpy(), ref, size, reach


def check(got, ref, size, reach, C):
    tol = f8_ref.linear_tolerance(ref, size, C, 0, False)
    # sums are fp32: at most a step of the least number (2^-149) for every term beside the relative bound; beyond fp32's largest number they are
    # infinite, or NaN where blocks of both signs are
    tol = tol - 1e-30 + (3 * -(-C // 128) + 1) * 2.0 ** -149
    assert not np.isfinite(got[np.abs(ref) - tol > 3.4028236e38]).any()
    sure = reach < 3.4028235e38 * (1 - 2.0 ** -20)  # (no order of the blocks leaves the range)
    assert np.isfinite(got[sure]).all()
    err = np.abs(got[sure] - ref[sure])
    assert (err <= tol[sure]).all(), float((err / tol[sure]).max())
    return sure.mean()


@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("ends", [(2.0 ** 63, 2.0 ** 63), (1.3 * 2.0 ** 120, 2.0 ** 6), (2.0 ** 6, 1.3 * 2.0 ** 120), (3e38, 1e-42), (1e-42, 3e38)])
def test_products_up_to_the_largest_number(ends, form, formats, w_block):
    M, K, C = form
    rng = np.random.default_rng(M + K)
    cb = -(-C // 128)
    xv = f8_ref.nearest(rng.standard_normal((M, C)) * 2.0 ** -3, formats[0])
    wv = f8_ref.nearest(rng.standard_normal((K, C)) * 2.0 ** -4, formats[1])
    xv[:, :128], wv[:, :128] = 0, 0  # a block whose sums are 0
    sx = (ends[0] * rng.uniform(0.5, 1, (cb, M))).astype(np.float32)
    sw = (ends[1] * rng.uniform(0.5, 1, (cb, K if w_block == 1 else -(-K // 128)))).astype(np.float32)
    sx[1, ::3] = 0
    sw[1, ::2] *= -1
    result = layer(xv, sx, wv, sw, w_block, *formats)
    assert check(*result, C) > 0


@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("formats", [("e4m3", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("ends", [(1e-20, 1e-17), (1e-17, 1e-20), (1.5 * 2.0 ** -100, 2.0 ** -24), (2.0 ** -24, 1.5 * 2.0 ** -100), (1e-40, 1e4), (1e4, 1e-40)])
def test_products_down_to_the_least_normal_number(ends, form, formats, w_block):
    M, K, C = form
    rng = np.random.default_rng(M + C)
    cb = -(-C // 128)
    top = f8_ref.FMAX[formats[0]]
    xv = f8_ref.nearest(top * rng.uniform(-1, 1, (M, C)), formats[0])
    wv = f8_ref.nearest(top * rng.uniform(0.5, 1, (K, C)), formats[1])
    sx = (ends[0] * rng.uniform(0.5, 1, (cb, M))).astype(np.float32)
    sw = (ends[1] * rng.uniform(0.5, 1, (cb, K if w_block == 1 else -(-K // 128)))).astype(np.float32)
    result = layer(xv, sx, wv, sw, w_block, *formats)
    assert check(*result, C) > 0


@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("form", FORMS)
def test_blocks_of_zeros_with_the_least_scale(form, w_block):
    # what sgs_quantize_f8 writes for them, 2^-126, beside scales of the usual sizes and on both sides at once: they add 0
    M, K, C = form
    rng = np.random.default_rng(C)
    cb = -(-C // 128)
    xv = f8_ref.nearest(rng.standard_normal((M, C)) * 50, "e4m3")
    wv = f8_ref.nearest(rng.standard_normal((K, C)) * 50, "e4m3")
    sx = (2.0 ** rng.integers(-30, -5, (cb, M))).astype(np.float32)
    sw = (2.0 ** rng.integers(-30, -5, (cb, K if w_block == 1 else -(-K // 128)))).astype(np.float32)
    xv[: M // 2, 128:256] = 0
    sx[1, : M // 2] = 2.0 ** -126
    wv[:, :128] = 0
    sw[0] = 2.0 ** -126
    xv[M // 3:, :128] = 0
    sx[0, M // 3:] = 2.0 ** -126
    result = layer(xv, sx, wv, sw, w_block, "e4m3", "e4m3")
    assert check(*result, C) == 1
