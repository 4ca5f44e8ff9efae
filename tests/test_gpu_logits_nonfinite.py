"""Distillation of rows with NaN, infinities and masks, in every form that a row may take (a warp, a block, the blocks of a cluster), against
64 bits."""
import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests import f8_ref
from tests.test_gpu_f8_layer import DT, stream
from tests.test_gpu_logits import lists

pytestmark = pytest.mark.gpu

# a warp a row; blocks of 256 threads; of 512; clusters of two and of eight
FORMS = [(1300, 700, 20), (13, 600, 20), (300, 30000, 20), (13, 30000, 20), (13, 131075, 40)]


def odd_rows(M, V, k, dtype, seed=11):
    """Logits and lists whose first 13 rows are the odd ones."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = 3 * torch.randn((M, V), generator=g, device="cuda")
    v, i = lists(g, z, k)
    nan, inf = float("nan"), float("inf")
    z[0], z[1], z[2], z[3] = -inf, nan, -inf, -inf   # nothing but minus infinity and a NaN: in the middle (and named), everywhere,
    z[0, V // 2], z[2, 0], z[3, V - 1] = nan, nan, nan  # first and last
    i[0, 1] = V // 2
    z[4, V // 3] = nan                               # a NaN next to ordinary logits
    z[5, V // 3] = inf
    z[6], z[6, 1] = -inf, inf
    z[7] = -inf                                      # nothing left: no NaN either
    z[8, V // 2:] = torch.finfo(dtype).min
    v[10, 2] = inf                                   # the teacher's own
    v[11, 2] = nan
    i[12] = -1                                       # no list: loss and gradient 0 whatever the logits
    z[12, V // 4] = nan
    return z.to(dtype), v, i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_rows_of_nan_and_infinities(form, dtype):
    (M, V, k), T = form, 2.0
    bf16 = dtype == "bf16"
    z, v, i = odd_rows(M, V, k, DT[dtype][1])
    d = sgs.DistillDesc(rows=M, classes=V, top=k, dtype=DT[dtype][0], temperature=T, grad_scale=1.0)
    zh, vh, ih = z.double().cpu().numpy(), v.cpu().numpy(), i.cpu().numpy()
    with np.errstate(invalid="ignore"):
        loss, stat, dz, Q, P = f8_ref.distill(zh, vh, ih, T, np.ones(M))
        # (the teacher's NaN and infinity enter no finite result: the tolerances are those of the other numbers)
        tol = np.nan_to_num(f8_ref.distill_tolerance(zh, np.where(np.isfinite(vh), vh, 0), ih, T), nan=0.0, posinf=0.0)
    # a teacher's NaN is a slot in use (the 64-bit statement leaves such slots out), and infinity less infinity is one: every probability
    # of those lists is NaN
    loss[10:12] = np.nan
    loss = np.where(loss > 3.4028235e38, np.inf, loss)  # (a mask of the type's lowest value, named by the teacher)
    dz[11] = Q[11] * T
    dz[11, ih[11]] = np.nan
    assert np.isnan(loss[[0, 1, 2, 3, 4, 5, 6, 10, 11]]).all() and loss[7] == np.inf and loss[12] == 0
    gl, gs = torch.full((M,), -7.0, device="cuda"), torch.full((M, 2), -7.0, device="cuda")
    for mode in ("loss", "step", "backward"):
        out = torch.full((M, V), -7.0, dtype=z.dtype, device="cuda")
        if mode == "backward":
            sgs.distill_backward(d, z.data_ptr(), v.data_ptr(), i.data_ptr(), gs.data_ptr(), 0, out.data_ptr(), stream())
        else:
            sgs.distill(d, z.data_ptr(), v.data_ptr(), i.data_ptr(), 0, gl.data_ptr(), gs.data_ptr(), out.data_ptr() if mode == "step" else 0, stream())
        torch.cuda.synchronize()
        if mode != "backward":
            got = gl.double().cpu().numpy()
            fine = np.isfinite(loss)
            np.testing.assert_array_equal(got[~fine], loss[~fine])
            assert (np.abs(got[fine] - loss[fine]) <= (T * T * tol * (1 + np.abs(loss) / (T * T)))[fine]).all()
            got = gs.double().cpu().numpy()
            np.testing.assert_array_equal(got[:, 0], stat[:, 0])
            fine = np.isfinite(stat[:, 1])
            np.testing.assert_array_equal(got[~fine, 1], stat[~fine, 1])
            assert (np.abs(got[fine, 1] - stat[fine, 1]) <= 2.0 ** -24 * (64 + V / 256) * (1 + np.abs(stat[fine, 1]))).all()
        if mode != "loss":
            got = out.double().cpu().numpy()
            np.testing.assert_array_equal(np.isnan(got), np.isnan(dz))
            # (roundings of an exponent of the size of the row's spread count relative to q, as everywhere)
            with np.errstate(invalid="ignore"):
                spread = np.nan_to_num(np.where(np.isfinite(zh), zh.max(1, keepdims=True) - zh, 0) / T, nan=0.0, posinf=0.0)
                bound = T * np.nan_to_num(Q + P) * (tol[:, None] + 2.0 ** -24 * 8 * spread) + 1e-37
            if bf16:
                bound = bound + 2.0 ** -8 * (np.abs(np.nan_to_num(dz)) + bound)
            err = np.where(np.isnan(dz), 0, np.abs(np.nan_to_num(got) - np.nan_to_num(dz)))
            assert (err <= bound).all(), (mode, np.unravel_index((err / bound).argmax(), err.shape))
