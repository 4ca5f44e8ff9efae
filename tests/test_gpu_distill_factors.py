"""The factor of the distillation gradient, grad_scale * row_scale * temperature, where a product of two of them leaves fp32's range and
that of all three does not."""
import pytest
import torch

from tests.test_gpu_f8_layer import DT
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
