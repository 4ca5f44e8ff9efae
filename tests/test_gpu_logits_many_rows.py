"""As many rows as the descriptors can name."""
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests.test_gpu_f8_layer import stream

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
