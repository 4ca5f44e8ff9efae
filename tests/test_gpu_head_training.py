"""The 8-bit layer and the operators on logits together, as they are used: the classifier in 8 bits taught by its full-precision form, with
both of its gradients, eager and as a captured graph; and the divergence of SubNets from the largest one as the scheduler's accuracy."""
import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from paper_2306_17266_b200 import workload as wl
from tests import f8_ref
from tests.gpu_util import gpu_forward, nets

pytestmark = pytest.mark.gpu


class Head:
    """Student classifier: x [M][C] bf16, weights [K][C] bf16; the teacher's logits come from the library's bf16 linear layer on its own x."""

    def __init__(self, M, C, K, top, T):
        g = torch.Generator(device="cuda").manual_seed(M + K)
        self.M, self.C, self.K, self.top, self.T = M, C, K, top, T
        self.x32 = torch.randn((M, C), generator=g, device="cuda")
        self.x = self.x32.to(torch.bfloat16)
        self.w = (torch.randn((K, C), generator=g, device="cuda") / C ** 0.5).to(torch.bfloat16)
        self.bias = 0.1 * torch.randn(K, generator=g, device="cuda")
        r16 = lambda n: (n + 15) // 16 * 16  # noqa: E731
        nb = lambda n: (n + 127) // 128  # noqa: E731
        u8 = lambda r, c: torch.zeros((r, r16(c)), dtype=torch.uint8, device="cuda")  # noqa: E731
        f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
        self.xq, self.xs, self.xqt, self.xst = u8(M, C), f(nb(C), M), u8(C, M), f(nb(M), C)
        self.wq, self.ws, self.wqt, self.wst = u8(K, C), f(nb(C), nb(K)), u8(C, K), f(nb(K), nb(C))
        self.gq, self.gs, self.gqt, self.gst = u8(M, K), f(nb(K), M), u8(K, M), f(nb(M), K)
        self.teach, self.z, self.dz = f(M, K), f(M, K), f(M, K)
        self.values, self.index = f(M, top), torch.zeros((M, top), dtype=torch.int32, device="cuda")
        self.loss, self.stat, self.dx, self.dw = f(M), f(M, 2), f(M, C), f(K, C)
        torch.cuda.synchronize()

    def step(self, st):
        M, C, K, top = self.M, self.C, self.K, self.top
        p = lambda t: t.data_ptr()  # noqa: E731
        sgs.aux_op([sgs.AuxDesc(kind=2, dtype=sgs.SGS_BF16, N=M, H=1, W=1, C=C, K=K, ld=C)],
                   [sgs.AuxArgs(x=p(self.x32), y=p(self.teach), w=p(self.w), bias=p(self.bias))], stream=st)
        sgs.top_logits(sgs.TopLogitsDesc(rows=M, classes=K, top=top, dtype=sgs.SGS_F32), p(self.teach), p(self.values), p(self.index), st)
        sgs.quantize_f8(sgs.QuantizeF8Desc(rows=M, cols=C, dtype=sgs.SGS_BF16, block_rows=1), p(self.x), p(self.xq), p(self.xs), p(self.xqt), p(self.xst), st)
        sgs.quantize_f8(sgs.QuantizeF8Desc(rows=K, cols=C, dtype=sgs.SGS_BF16, block_rows=128), p(self.w), p(self.wq), p(self.ws), p(self.wqt), p(self.wst), st)
        sgs.linear_f8(sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=K, Cmax=C, w_block_rows=128, y_dtype=sgs.SGS_F32), p(self.xq), p(self.xs), p(self.wq), p(self.ws),
                      p(self.bias), p(self.z), st)
        sgs.distill(sgs.DistillDesc(rows=M, classes=K, top=top, dtype=sgs.SGS_F32, temperature=self.T, grad_scale=1.0 / M), p(self.z), p(self.values),
                    p(self.index), 0, p(self.loss), p(self.stat), p(self.dz), st)
        sgs.quantize_f8(sgs.QuantizeF8Desc(rows=M, cols=K, dtype=sgs.SGS_F32, format=sgs.SGS_E5M2, block_rows=1), p(self.dz), p(self.gq), p(self.gs), p(self.gqt),
                        p(self.gst), st)
        sgs.linear_f8(sgs.LinearF8Desc(M=M, K=C, C=K, Kmax=C, Cmax=K, x_format=sgs.SGS_E5M2, w_block_rows=128, y_dtype=sgs.SGS_F32), p(self.gq), p(self.gs),
                      p(self.wqt), p(self.wst), 0, p(self.dx), st)
        sgs.linear_f8(sgs.LinearF8Desc(M=K, K=C, C=M, Kmax=C, Cmax=M, x_format=sgs.SGS_E5M2, w_block_rows=1, y_dtype=sgs.SGS_F32), p(self.gqt), p(self.gst),
                      p(self.xqt), p(self.xst), 0, p(self.dw), st)

    def outputs(self):
        return [t.clone() for t in (self.values, self.index, self.z, self.loss, self.stat, self.dz, self.dx, self.dw)]


@pytest.mark.parametrize("M,C,K,top,T", [(64, 512, 1000, 32, 2.0), (150, 300, 333, 20, 1.0), (1, 2048, 1000, 5, 4.0)])
def test_head_taught_by_its_full_precision_form(M, C, K, top, T):
    h = Head(M, C, K, top, T)
    h.step(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert sgs.device_status() == 0
    n = lambda t: t.double().cpu().numpy()  # noqa: E731
    # teacher: fp32 sums of bf16 weights; the list is that of the logits it was taken from
    teach = n(h.x32) @ n(h.w).T + n(h.bias)
    assert np.abs(n(h.teach) - teach).max() <= 1e-5 * np.abs(teach).max()
    np.testing.assert_array_equal(h.index.cpu().numpy(), f8_ref.top(n(h.teach), top))

    def check(got, xm, ws_, ref_scales, xs, w_block, bias, rows, cols, red):
        ref, size = f8_ref.linear(xm, xs, ws_, ref_scales, w_block, bias, 0, rows, cols, red)
        assert (np.abs(n(got) - ref) <= f8_ref.linear_tolerance(ref, size, red, 0, False)).all()
    xv, xs = f8_ref.quantize(n(h.x), "e4m3", 1)
    wv, ws = f8_ref.quantize(n(h.w), "e4m3", 128)
    check(h.z, xv, wv, ws, xs, 128, n(h.bias), M, K, C)
    loss, stat, dz, Q, P = f8_ref.distill(n(h.z), n(h.values), h.index.cpu().numpy(), T, np.full(M, 1.0 / M))
    tol = f8_ref.distill_tolerance(n(h.z), n(h.values), h.index.cpu().numpy(), T)
    assert (np.abs(n(h.loss) - loss) <= T * T * tol * (1 + loss / (T * T))).all()
    assert (np.abs(n(h.dz) - dz) <= T / M * (Q + P) * tol[:, None] + 1e-37).all()
    gv, gs = f8_ref.quantize(n(h.dz), "e5m2", 1)
    wtv, wts = f8_ref.quantize(n(h.w).T, "e4m3", 128)
    check(h.dx, gv, wtv, wts, gs, 128, None, M, C, K)
    gtv, gts = f8_ref.quantize(n(h.dz).T, "e5m2", 1)
    xtv, xts = f8_ref.quantize(n(h.x).T, "e4m3", 1)
    check(h.dw, gtv, xtv, xts, gts, 1, None, K, C, M)


def test_the_same_step_captured_and_on_two_streams():
    h = Head(96, 256, 520, 16, 2.0)
    st = torch.cuda.Stream()
    h.step(st.cuda_stream)
    st.synchronize()
    first = h.outputs()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        h.step(st.cuda_stream)
    other, st2 = Head(96, 256, 520, 16, 2.0), torch.cuda.Stream()
    for t in (h.z, h.dz, h.dx, h.dw, h.loss):
        t.zero_()
    torch.cuda.synchronize()
    for _ in range(5):  # two at a time: nothing is shared between calls
        with torch.cuda.stream(st):
            g.replay()
        other.step(st2.cuda_stream)
    torch.cuda.synchronize()
    for a, b, c in zip(first, h.outputs(), other.outputs()):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("family,res,bf16", [(wl.TINY, 32, False), (wl.RESNET, 64, True)])
def test_divergence_of_subnets_and_the_scheduler(family, res, bf16):
    blob, onet, gnet = nets(family, bf16)
    cfgs = wl.uniform_stream(family, 4, seed=9) + [wl.extreme_cfg(family, True)]
    teacher = wl.extreme_cfg(family, True)
    x = wl.make_inputs(1, 6, res, seed=3, bf16=bf16).reshape(6, res, res, 3)
    dx = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    dx = dx.to(torch.bfloat16) if bf16 else dx
    top, T = min(5, gnet.n_classes), 2.0
    before = gnet.cache_stats().as_dict()
    got = gnet.subnet_divergence(teacher, cfgs, dx.data_ptr(), 6, res, top, T, torch.cuda.current_stream().cuda_stream)
    assert gnet.cache_stats().as_dict() == {**before, "device_bytes_allocated": gnet.cache_stats().device_bytes_allocated}
    t = gpu_forward(gnet, teacher, x, bf16).astype(np.float64)
    index = f8_ref.top(t, top).astype(np.int32)
    values = np.take_along_axis(t, index, 1).astype(np.float32)
    for cfg, d in zip(cfgs, got):
        z = gpu_forward(gnet, cfg, x, bf16).astype(np.float64)
        loss = f8_ref.distill(z, values, index, T, np.ones(6))[0]
        tol = T * T * f8_ref.distill_tolerance(z, values, index, T) * (1 + loss)
        assert abs(d - loss.mean()) <= tol.mean()
    # minus the divergence is an accuracy: the most accurate SubNet is the nearest to the teacher
    gnet.cache_set_candidates(cfgs[:2])
    sched = sgs.Scheduler(gnet, cfgs, -got, 4)
    rows, _ = sched.step([sgs.SGS_STRICT_LATENCY], [0.0], [1.0])
    assert rows[0] == int(np.argmin(got))
    sched.close()
    gnet.cache_set_candidates([])
    for kw in (dict(top=0), dict(top=gnet.n_classes + 1), dict(temperature=0.0), dict(temperature=float("nan"))):
        with pytest.raises(sgs.SgsError) as e:
            gnet.subnet_divergence(teacher, cfgs, dx.data_ptr(), 6, res, **{**dict(top=top, temperature=T), **kw})
        assert e.value.status == sgs.binding.SGS_EINVAL
    gnet.set_option("fail_alloc_after", 0)
    with pytest.raises(sgs.SgsError) as e:
        gnet.subnet_divergence(teacher, cfgs, dx.data_ptr(), 6, res, top, T)
    gnet.set_option("fail_alloc_after", -1)
    assert e.value.status == sgs.binding.SGS_ENOMEM
    again = gnet.subnet_divergence(teacher, cfgs, dx.data_ptr(), 6, res, top, T, torch.cuda.current_stream().cuda_stream)
    np.testing.assert_array_equal(got, again)
