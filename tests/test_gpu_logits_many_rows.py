"""As many rows as the descriptors can name, and rows that lie far apart."""
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests.test_gpu_f8_layer import stream
from tests.test_gpu_logits import lists, run_distill

pytestmark = pytest.mark.gpu


def test_distill_of_two_to_the_31_less_one_rows():
    # one class, one slot: q = p = 1, so every loss is 0 whatever the logits
    M = 2 ** 31 - 1
    z = torch.empty(M, dtype=torch.bfloat16, device="cuda").fill_(3)
    teacher, index = torch.empty(M, device="cuda").fill_(1), torch.zeros(M, dtype=torch.int32, device="cuda")
    loss = torch.empty(M, device="cuda").fill_(-7)
    index[-2] = -1  # (no list: 0 as well)
    z[-1] = float("inf")
    d = sgs.DistillDesc(rows=M, classes=1, top=1, dtype=sgs.SGS_BF16, temperature=1.0, grad_scale=1.0)
    sgs.distill(d, z.data_ptr(), teacher.data_ptr(), index.data_ptr(), 0, loss.data_ptr(), 0, 0, stream())
    assert torch.isnan(loss[-1]) and not torch.isnan(loss[:-1]).any()
    assert int(torch.count_nonzero(loss[:-1])) == 0
    del z, teacher, index, loss
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_in_the_place_of_rows_that_lie_far_apart(dtype):
    # element offsets up to 2.4e9; the bound is relative to q and p
    pitch, M, V = 1 << 28, 10, 3000
    g = torch.Generator(device="cuda").manual_seed(1)
    big = torch.empty((M, pitch), dtype=dtype, device="cuda")
    z = big[:, :V]
    z.copy_(3 * torch.randn((M, V), generator=g, device="cuda"))
    v, i = lists(g, z, 20, ragged=True)
    run_distill(z, v, i, 2.0, torch.rand(M, generator=g, device="cuda"), in_place=True)
    del big, z
    torch.cuda.empty_cache()
