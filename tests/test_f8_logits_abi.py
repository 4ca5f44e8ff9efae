"""CPU-side checks of the 8-bit floating point layers and the operators on logits: refusals before any device is touched, and the
64-bit statements that the GPU tests compare with, against hand values, torch and differences."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests import f8_ref

EINVAL, EUNSUPPORTED = sgs.binding.SGS_EINVAL, sgs.binding.SGS_EUNSUPPORTED
P = 1 << 20  # an address that is never read


def test_struct_sizes():
    assert ctypes.sizeof(sgs.QuantizeF8Desc) == 40 and ctypes.sizeof(sgs.LinearF8Desc) == 60
    assert ctypes.sizeof(sgs.TopLogitsDesc) == 24 and ctypes.sizeof(sgs.DistillDesc) == 36


def test_null_arguments():
    L = sgs.lib()
    assert L.sgs_quantize_f8(None, P, P, P, P, P, None) == EINVAL
    assert L.sgs_linear_f8(None, P, P, P, P, P, P, None) == EINVAL
    assert L.sgs_top_logits(None, P, P, P, None) == EINVAL
    assert L.sgs_distill(None, P, P, P, P, P, P, P, None) == EINVAL
    assert L.sgs_distill_backward(None, P, P, P, P, P, P, None) == EINVAL
    q = sgs.QuantizeF8Desc(rows=1, cols=1, block_rows=1)
    for args in ((None, P, P, P, P), (P, None, P, P, P), (P, P, None, P, P), (P, P, P, None, P), (P, P, P, P, None), (P, None, None, None, None)):
        assert L.sgs_quantize_f8(ctypes.byref(q), *args, None) == EINVAL
    d = sgs.DistillDesc(rows=1, classes=1, top=1, temperature=1.0)
    assert L.sgs_distill(ctypes.byref(d), P, P, P, None, None, P, P, None) == EINVAL
    assert L.sgs_distill_backward(ctypes.byref(d), P, P, P, None, None, P, None) == EINVAL
    assert L.sgs_distill_backward(ctypes.byref(d), P, P, P, P, None, None, None) == EINVAL


@pytest.mark.parametrize("change,status", [
    (dict(M=0), EINVAL), (dict(K=0), EINVAL), (dict(C=0), EINVAL), (dict(K=65), EINVAL), (dict(C=65), EINVAL), (dict(x_format=2), EINVAL), (dict(w_format=-1), EINVAL),
    (dict(w_block_rows=0), EINVAL), (dict(y_dtype=2), EINVAL), (dict(act=3), EINVAL), (dict(ldx=48), EINVAL), (dict(ldw=48), EINVAL), (dict(ldy=63), EINVAL),
    (dict(ldsx=7), EINVAL), (dict(ldsw=63), EINVAL), (dict(ldx=-64), EINVAL), (dict(ldx=72), EUNSUPPORTED), (dict(ldw=72), EUNSUPPORTED),
    (dict(M=2 ** 31 - 100), EUNSUPPORTED), (dict(M=2 ** 30, K=2 ** 30, Kmax=2 ** 30), EUNSUPPORTED)])
def test_linear_refusals(change, status):
    d = sgs.LinearF8Desc(**{**dict(M=8, K=64, C=64, Kmax=64, Cmax=64, w_block_rows=1), **change})
    assert sgs.lib().sgs_linear_f8(ctypes.byref(d), P, P, P, P, None, P, None) == status


def test_addresses_that_no_device_owns_are_refused():
    # (with a device or without one: nothing is launched)
    d = sgs.LinearF8Desc(M=8, K=64, C=64, Kmax=64, Cmax=64, w_block_rows=1)
    assert sgs.lib().sgs_linear_f8(ctypes.byref(d), P, P, P, P, None, P, None) == EINVAL
    assert sgs.lib().sgs_linear_f8(ctypes.byref(d), P + 8, P, P, P, None, P, None) == EUNSUPPORTED
    assert sgs.lib().sgs_linear_f8(ctypes.byref(d), P, P + 2, P, P, None, P, None) == EINVAL
    t = sgs.TopLogitsDesc(rows=8, classes=64, top=3)
    assert sgs.lib().sgs_top_logits(ctypes.byref(t), P, P, P, None) == EINVAL


@pytest.mark.parametrize("change", [dict(rows=0), dict(cols=-1), dict(dtype=3), dict(format=2), dict(block_rows=64), dict(ldx=9), dict(ldq=9), dict(ldqt=7),
                                    dict(lds=7), dict(ldst=9), dict(ldq=-16)])
def test_quantize_refusals(change):
    d = sgs.QuantizeF8Desc(**{**dict(rows=8, cols=10, block_rows=1), **change})
    assert sgs.lib().sgs_quantize_f8(ctypes.byref(d), P, P, P, P, P, None) == EINVAL


def test_decode_and_rounding_of_the_statements():
    every = np.arange(256, dtype=np.uint8)
    for fmt, t in (("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)):
        mine, theirs = f8_ref.decode(every, fmt), torch.from_numpy(every.copy()).view(t).double().numpy()
        np.testing.assert_array_equal(mine, theirs)
        v = np.concatenate([np.linspace(-f8_ref.FMAX[fmt], f8_ref.FMAX[fmt], 4001), np.linspace(-0.1, 0.1, 4001), 2.0 ** -np.arange(30)]).astype(np.float32)
        np.testing.assert_array_equal(f8_ref.nearest(v.astype(np.float64), fmt), torch.from_numpy(v).to(t).double().numpy())
    assert f8_ref.scale_for(448.0, "e4m3") == 1.0 and f8_ref.scale_for(448.1, "e4m3") == 2.0 and f8_ref.scale_for(0, "e4m3") == 2.0 ** -126
    assert f8_ref.scale_for(224.0, "e4m3") == 0.5 and f8_ref.scale_for(57345.0, "e5m2") == 2.0


def test_distill_statement_against_torch_and_differences():
    rng = np.random.default_rng(3)
    z, k, T = 2 * rng.standard_normal((4, 30)), 6, 1.5
    index = np.argsort(-z + rng.standard_normal(z.shape), 1)[:, :k].astype(np.int32)
    teacher = rng.standard_normal((4, k)).astype(np.float32)
    index[1, 3:] = -1
    index[2, :] = 30
    index[3, 1] = index[3, 0]
    coef = np.array([1.0, 2.0, 3.0, 0.5])
    loss, stat, dz, _, _ = f8_ref.distill(z, teacher, index, T, coef)
    assert loss[2] == 0 and not dz[2].any()
    zt = torch.from_numpy(z).requires_grad_()
    total = 0
    for r in (0, 1, 3):
        use = index[r] >= 0
        p = torch.softmax(torch.from_numpy(teacher[r][use]).double() / T, 0)
        lq = torch.log_softmax(zt[r] / T, 0)[torch.from_numpy(index[r][use].astype(np.int64))]
        l = T * T * (p * (p.log() - lq)).sum()
        assert abs(float(l) - loss[r]) < 1e-12
        total = total + coef[r] * l
    total.backward()
    np.testing.assert_allclose(dz, zt.grad.numpy(), atol=1e-12)
    for r, c in ((0, 3), (1, int(index[1, 0])), (3, int(index[3, 0])), (2, 5)):
        up, down = z.copy(), z.copy()
        up[r, c] += 1e-5
        down[r, c] -= 1e-5
        slope = (f8_ref.distill(up, teacher, index, T, coef)[0][r] - f8_ref.distill(down, teacher, index, T, coef)[0][r]) / 2e-5
        assert abs(coef[r] * slope - dz[r, c]) < 1e-8


def test_top_statement():
    z = np.array([[1.0, 3.0, 3.0, -np.inf, np.nan, 0.0, -0.0]])
    assert list(f8_ref.top(z, 7)[0]) == [4, 1, 2, 0, 5, 6, 3]
