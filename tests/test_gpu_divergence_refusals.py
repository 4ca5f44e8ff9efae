"""What sgs_subnet_divergence refuses, and what it leaves as it was then."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from paper_2306_17266_b200 import workload as wl
from tests.gpu_util import nets

pytestmark = pytest.mark.gpu

RES, BATCH = 32, 3


def setup():
    _, _, gnet = nets(wl.TINY, False)
    cfgs = wl.uniform_stream(wl.TINY, 3, seed=5)
    x = torch.from_numpy(np.ascontiguousarray(wl.make_inputs(1, BATCH, RES, seed=3).reshape(BATCH, RES, RES, 3))).cuda()
    return gnet, wl.extreme_cfg(wl.TINY, True), cfgs, x


def refused(status, gnet, *args, **kw):
    with pytest.raises(sgs.SgsError) as e:
        gnet.subnet_divergence(*args, **kw)
    assert e.value.status == status


def test_a_captured_stream_is_refused_and_the_capture_goes_on():
    gnet, teacher, cfgs, x = setup()
    want = gnet.subnet_divergence(teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0, torch.cuda.current_stream().cuda_stream)
    y = torch.zeros(8, device="cuda")
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        y.add_(1)
        refused(sgs.binding.SGS_EINVAL, gnet, teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0, st.cuda_stream)
        y.add_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert (y == 2).all()
    np.testing.assert_array_equal(gnet.subnet_divergence(teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0, st.cuda_stream), want)


def test_queries_without_logits_are_refused():
    gnet, teacher, cfgs, x = setup()
    gnet.set_option("stop_after_layer", 1)
    try:
        refused(sgs.binding.SGS_EINVAL, gnet, teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0)
    finally:
        gnet.set_option("stop_after_layer", -1)
    assert np.isfinite(gnet.subnet_divergence(teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0)).all()


def test_configs_and_arguments_out_of_range():
    gnet, teacher, cfgs, x = setup()
    bad = wl.copy_cfg(cfgs[0])
    bad.width[2] = 0.6
    before = gnet.get_counter("kernel_launches")
    refused(sgs.binding.SGS_ECONFIG, gnet, bad, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0)
    refused(sgs.binding.SGS_ECONFIG, gnet, teacher, cfgs + [bad], x.data_ptr(), BATCH, RES, 5, 2.0)
    for batch, res in ((0, RES), (-1, RES), (BATCH, 4), (BATCH, 2000)):
        refused(sgs.binding.SGS_EINVAL, gnet, teacher, cfgs, x.data_ptr(), batch, res, 5, 2.0)
    refused(sgs.binding.SGS_EINVAL, gnet, teacher, cfgs, 0, BATCH, RES, 5, 2.0)
    out, arr = np.full(3, -7.0), wl.cfg_array(cfgs)
    L = sgs.lib()
    args = [gnet._h, ctypes.byref(teacher), ctypes.addressof(arr), 3, x.data_ptr(), BATCH, RES, 5, 2.0, out.ctypes.data, None]
    for at, value in ((0, None), (1, None), (2, None), (3, 0), (3, -1), (9, None)):
        assert L.sgs_subnet_divergence(*[value if i == at else a for i, a in enumerate(args)]) == sgs.binding.SGS_EINVAL
    assert (out == -7).all() and gnet.get_counter("kernel_launches") == before


def test_a_wait_that_ran_out_is_reported():
    gnet, teacher, cfgs, x = setup()
    want = gnet.subnet_divergence(teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0)
    try:
        sgs.debug_expire_wait(1000, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        refused(sgs.binding.SGS_ETIMEOUT, gnet, teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0)
    finally:
        sgs.device_status_clear()
    np.testing.assert_array_equal(gnet.subnet_divergence(teacher, cfgs, x.data_ptr(), BATCH, RES, 5, 2.0), want)
