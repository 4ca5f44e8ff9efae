"""The bounded waits of the 8-bit float layer: weights that never arrive make the waits for them run out (limit 1 ms); every block returns, the
status word says so, what was written is right, and the next call is as before."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests.test_gpu_f8_layer import operand, stream

# split over a cluster, without one, with 64 rows a block; single tiles, several a block; pairs of blocks, several tiles a pair
FORMS = [(16, 200, 700), (8, 200, 300), (30, 1000, 2048), (64, 200, 1300), (200, 300, 600), (12544, 200, 300), (2600, 2700, 1111)]


@pytest.mark.gpu
@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("which", ["first", "third", "last"])
@pytest.mark.parametrize("form", FORMS)
def test_weights_that_never_arrive(form, which, w_block):
    M, K, C = form
    rng = np.random.default_rng(M)
    x, sx, _, _ = operand(rng, M, C, "e4m3", 1, 1.0)
    w, sw, _, _ = operand(rng, K, C, "e4m3", w_block, 0.1)
    d = sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=K, Cmax=C, w_block_rows=w_block, y_dtype=sgs.SGS_F32)
    args = (x.data_ptr(), sx.data_ptr(), w.data_ptr(), sw.data_ptr(), 0)
    y, late, again = (torch.full((M + 1, K), -7.0, device="cuda") for _ in range(3))
    sgs.linear_f8(d, *args, y.data_ptr(), stream())
    torch.cuda.synchronize()
    assert sgs.device_status() == 0
    block = {"first": 0, "third": 2, "last": (C + 127) // 128 - 1}[which]
    try:
        sgs.debug_expire_f8_wait(d, *args, late.data_ptr(), block, 1000, stream())
        torch.cuda.synchronize()  # returns: every block ended on its own
        assert sgs.device_status() != 0
    finally:
        sgs.device_status_clear()
    assert (late[M] == -7).all()
    if M > 64:  # (a cluster whose blocks share a reduction may have written anything)
        assert ((late == y) | (late == -7)).all()
    assert sgs.device_status() == 0
    for _ in range(3):
        sgs.linear_f8(d, *args, again.data_ptr(), stream())
    torch.cuda.synchronize()
    assert sgs.device_status() == 0 and torch.equal(again, y)


def test_refusals():
    P = 1 << 20  # (never read)
    call = lambda d, block, limit: sgs.lib().sgs_debug_expire_f8_wait(ctypes.byref(d) if d else None, P, P, P, P, None, P, block, limit, None)  # noqa: E731
    d = sgs.LinearF8Desc(M=8, K=64, C=300, Kmax=64, Cmax=300, w_block_rows=1)
    for block, limit in ((-1, 1000), (3, 1000), (0, 0), (0, 1000001)):
        assert call(d, block, limit) == sgs.binding.SGS_EINVAL
    assert call(None, 0, 1000) == sgs.binding.SGS_EINVAL
    d.K = 65
    assert call(d, 0, 1000) == sgs.binding.SGS_EINVAL
