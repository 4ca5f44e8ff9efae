"""Top logits of many short rows, where blocks of 128 threads take a row each: read element by element up to 2048 bf16 or 1024 fp32 logits,
as a stream of vectors beyond, up to 16 KB; and longer rows, which take blocks of 512."""
import pytest
import torch

from tests.test_gpu_f8_layer import DT
from tests.test_gpu_logits import run_top

pytestmark = pytest.mark.gpu


def rows(M, V, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.arange(V, device="cuda")
    z = 3 * torch.randn((M, V), generator=g, device="cuda")
    z[3] = 0                                  # many equal values: the k-th is found eight bits at a time
    z[4] = a % 3
    z[5, ::2] = float("nan")
    z[6] = float("-inf")
    z[7, V // 2:] = torch.finfo(dtype).min
    z[8] = a                                  # the largest at the end, at the start, in one thread's vectors
    z[9] = -a
    z[10, : V // 3] += 50
    z[11, (a // (16 // dtype.itemsize)) % 128 == 5] += 40
    z[12, ::7] = float("inf")
    z[13] = -0.0
    z[13, ::5] = 0.0
    z[14, V - 1], z[14, 0] = 1e30, 1e30       # the edges of the row
    big = torch.empty((M, V + pad), dtype=dtype, device="cuda")
    big[:, :V] = z.to(dtype)
    return big[:, :V]


BF16 = [(400, 1000), (600, 3), (296, 2048), (296, 2049), (300, 4099), (297, 8000), (296, 8192), (296, 8193)]
F32 = [(400, 1000), (600, 3), (296, 1024), (296, 1025), (300, 2051), (297, 4095), (296, 4096), (300, 4099), (297, 8000)]


@pytest.mark.parametrize("k", [1, 5, 64, 100])
@pytest.mark.parametrize("dtype,M,V", [("bf16", *s) for s in BF16] + [("f32", *s) for s in F32])
def test_many_short_rows(dtype, M, V, k):
    if V < 16:
        z = 3 * torch.randn((M, V), generator=torch.Generator(device="cuda").manual_seed(V), device="cuda")
        run_top(z.to(DT[dtype][1]), min(k, V))
        return
    run_top(rows(M, V, DT[dtype][1], V), k)


@pytest.mark.parametrize("k", [7, 64])
@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("dtype,V", [("bf16", 2050), ("bf16", 5001), ("f32", 1030), ("f32", 3001), ("bf16", 1999), ("f32", 777)])
def test_many_short_rows_at_odd_addresses(dtype, V, pad, k):
    run_top(rows(300, V, DT[dtype][1], V + pad, pad), k, ldt=k + 3)
