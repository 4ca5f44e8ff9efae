"""The factor of the distillation gradient, grad_scale * row_scale * temperature, where a product of two of them leaves fp32's range and
that of all three does not; and lists at a pitch of their own."""
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests.test_gpu_f8_layer import DT, stream
from tests.test_gpu_logits import lists, run_distill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,k", [(1300, 700, 20), (5, 600, 20), (5, 30000, 20)])
@pytest.mark.parametrize("grad_scale,row,T", [(1e38, 2e-38, 100.0), (1e-40, 1e38, 0.25), (-1e38, 1e-30, 50.0), (3e-39, 2e38, 1e-3)])
def test_factors_at_the_ends_of_their_range(M, V, k, grad_scale, row, T, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (min(T, 3.0) * torch.randn((M, V), generator=g, device="cuda")).to(DT[dtype][1])
    v, i = lists(g, z, k, ragged=True)
    if T < 1:
        v = (v * T).contiguous()
    row_scale = row * (0.5 + 0.5 * torch.rand(M, generator=g, device="cuda"))
    row_scale[::3] = 0  # g = 0: the gradient is 0
    outs = run_distill(z, v, i, T, row_scale, grad_scale)
    for dz in outs:
        assert (dz[::3] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,k,ldt", [(1300, 700, 20, 33), (5, 600, 200, 201), (5, 30000, 20, 64), (2, 131075, 150, 151)])
def test_lists_at_a_pitch_of_their_own(M, V, k, ldt, dtype):
    # what lies behind a list names classes and is not read
    g = torch.Generator(device="cuda").manual_seed(k)
    z = (3 * torch.randn((M, V), generator=g, device="cuda")).to(DT[dtype][1])
    v, i = lists(g, z, k, ragged=True)
    wide_v, wide_i = torch.full((M, ldt), 50.0, device="cuda"), torch.zeros((M, ldt), dtype=torch.int32, device="cuda")
    wide_v[:, :k], wide_i[:, :k] = v, i
    scale = torch.rand(M, generator=g, device="cuda")
    results = []
    for pitch, values, index in ((0, v, i), (ldt, wide_v, wide_i)):
        loss, stat, dz, back = (torch.full(s, -7.0, dtype=t, device="cuda") for s, t in (((M,), torch.float32), ((M, 2), torch.float32), ((M, V), z.dtype), ((M, V), z.dtype)))
        d = sgs.DistillDesc(rows=M, classes=V, top=k, ldt=pitch, dtype=DT[dtype][0], temperature=2.0, grad_scale=0.5)
        sgs.distill(d, z.data_ptr(), values.data_ptr(), index.data_ptr(), scale.data_ptr(), loss.data_ptr(), stat.data_ptr(), dz.data_ptr(), stream())
        sgs.distill_backward(d, z.data_ptr(), values.data_ptr(), index.data_ptr(), stat.data_ptr(), scale.data_ptr(), back.data_ptr(), stream())
        torch.cuda.synchronize()
        results.append((loss, stat, dz, back))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    run_distill(z, v, i, 2.0, scale, 0.5)
