"""Entry points as the first CUDA call of a host thread: the current context is not bound to the thread by then, and the results are those of
the thread that has made others."""
import threading

import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from paper_2306_17266_b200 import workload as wl
from tests.gpu_util import nets, to_device

pytestmark = pytest.mark.gpu

p = lambda t: t.data_ptr()  # noqa: E731
rand = lambda *s: torch.randn(s, generator=torch.Generator(device="cuda").manual_seed(sum(s)), device="cuda")  # noqa: E731
codes = lambda *s: torch.randint(0, 0x70, s, generator=torch.Generator(device="cuda").manual_seed(sum(s)), device="cuda", dtype=torch.uint8)  # noqa: E731


def both(call, outs):
    """call() in a thread of its own, then in this one: the outputs of the two."""
    torch.cuda.synchronize()
    errors = []

    def work():
        try:
            call()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    first = [o.clone() for o in outs]
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    call()
    torch.cuda.synchronize()
    for a, b in zip(first, outs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and a.view(torch.uint8).any()


@pytest.mark.parametrize("M,K,C", [(3, 203, 707), (40, 131, 2000), (207, 301, 300), (2601, 2700, 1111)])
def test_linear_f8(M, K, C):
    r16 = (C + 15) // 16 * 16
    x, w = codes(M, r16), codes(K, r16)
    sx, sw, y = torch.ones(((C + 127) // 128, M), device="cuda"), torch.ones(((C + 127) // 128, K), device="cuda"), torch.zeros((M, K), device="cuda")
    d = sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=K, Cmax=C, w_block_rows=1, y_dtype=sgs.SGS_F32)
    both(lambda: sgs.linear_f8(d, p(x), p(sx), p(w), p(sw), 0, p(y)), [y])


def test_quantize_f8():
    x, q, s = rand(100, 300), torch.zeros((100, 304), dtype=torch.uint8, device="cuda"), torch.zeros((3, 100), device="cuda")
    both(lambda: sgs.quantize_f8(sgs.QuantizeF8Desc(rows=100, cols=300, dtype=sgs.SGS_F32, block_rows=1), p(x), p(q), p(s)), [q, s])


def test_operators_on_logits():
    z, v, i = rand(7, 40001), torch.zeros((7, 9), device="cuda"), torch.zeros((7, 9), dtype=torch.int32, device="cuda")
    both(lambda: sgs.top_logits(sgs.TopLogitsDesc(rows=7, classes=40001, top=9, dtype=sgs.SGS_F32), p(z), p(v), p(i)), [v, i])
    loss, stat, dz = torch.zeros(7, device="cuda"), torch.zeros((7, 2), device="cuda"), torch.zeros((7, 40001), device="cuda")
    d = sgs.DistillDesc(rows=7, classes=40001, top=9, dtype=sgs.SGS_F32, temperature=2.0, grad_scale=1.0)
    z2 = rand(7, 40001) + 0.1 * rand(1, 40001)
    both(lambda: sgs.distill(d, p(z2), p(v), p(i), 0, p(loss), p(stat), p(dz)), [loss, stat, dz])
    both(lambda: sgs.distill_backward(d, p(z2), p(v), p(i), p(stat), 0, p(dz)), [dz])


@pytest.mark.parametrize("static", [False, True])
def test_convolution_layers(static):
    N, H, C, K, k = 1, 13, 72, 136, 3
    x, w = rand(N, H, H, C).to(torch.bfloat16), (0.05 * rand(K, k, k, C)).to(torch.bfloat16)
    one, zero, y = torch.ones(K, device="cuda"), torch.zeros(K, device="cuda"), torch.zeros((N, H, H, K), dtype=torch.bfloat16, device="cuda")
    d = sgs.ConvDesc(N=N, H=H, W=H, C=C, K=K, Kmax=K, Cmax=C, R=k, k=k, stride=1, act=1, dtype=sgs.SGS_BF16)
    f = sgs.conv2d_sliced_static if static else sgs.conv2d_sliced
    both(lambda: f(d, p(x), p(w), p(one), p(zero), 0, p(y)), [y])


def test_int8_layer():
    N, H, C, K = 1, 11, 80, 144
    x, w = codes(N, H, H, C), codes(K, 1, 1, C)
    mult, shift, bias = torch.full((K,), 1 << 30, dtype=torch.int32, device="cuda"), torch.full((K,), 8, dtype=torch.int32, device="cuda"), torch.zeros(K, dtype=torch.int32, device="cuda")
    y = torch.zeros((N, H, H, K), dtype=torch.uint8, device="cuda")
    d = sgs.ConvI8Desc(N=N, H=H, W=H, C=C, K=K, Kmax=K, Cmax=C, R=1, k=1, stride=1, relu=0)
    both(lambda: sgs.conv2d_sliced_i8(d, p(x), p(w), p(mult), p(shift), p(bias), 0, p(y)), [y])


def test_linear_of_the_other_layers():
    x, w, bias, y = rand(9, 200), rand(130, 200).to(torch.bfloat16), rand(130), torch.zeros((9, 130), device="cuda")
    both(lambda: sgs.aux_op([sgs.AuxDesc(kind=2, dtype=sgs.SGS_BF16, N=9, H=1, W=1, C=200, K=130, ld=200)], [sgs.AuxArgs(x=p(x), y=p(y), w=p(w), bias=p(bias))]), [y])


@pytest.mark.parametrize("family,bf16", [(wl.RESNET, True), (wl.MBV3, True), (wl.TINY, False)])
def test_queries_streams_and_divergence(family, bf16):
    # SubNets and sizes of this test's own: their plans are made in the other thread, and use the same kernels
    _, _, gnet = nets(family, bf16)
    n, res = 4, 72
    cfgs = wl.uniform_stream(family, n, seed=7171)
    x = to_device(wl.make_inputs(n, 1, res, seed=9, bf16=bf16).reshape(n, res, res, 3), bf16)
    out = torch.zeros((n, gnet.n_classes), device="cuda")
    before = gnet.get_counter("tc_convs")
    both(lambda: gnet.subnet_run(cfgs[0], p(x), n, res, p(out)), [out])
    launched = gnet.get_counter("tc_convs") - before
    assert launched % 2 == 0  # (as many in the one as in the other)
    st = torch.cuda.Stream()
    opts = sgs.StreamOpts(cache_enabled=1, window_q=2, concurrency=2, wave=2)
    both(lambda: gnet.stream_run(cfgs, p(x), 1, res, p(out), opts, st.cuda_stream), [out])
    got = []
    both(lambda: got.append(gnet.subnet_divergence(cfgs[1], cfgs, p(x), n, res, 3, 2.0)), [])
    np.testing.assert_array_equal(got[0], got[1])
