"""Edges of the 8-bit float layers and of the operators on logits: the forms that many rows take, several tiles a block, outputs that start
anywhere, offsets beyond 32 bits, host threads."""
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests import f8_ref
from tests.test_gpu_f8_layer import DT, check_side, operand, quantize, run_linear, stream
from tests.test_gpu_logits import lists, run_distill, run_top

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,k", [(1300, 700, 20), (1200, 1000, 128), (1184, 2048, 1), (1500, 9, 9), (1190, 1000, 129)])
def test_distill_many_short_rows(M, V, k, dtype):
    # a warp a row (but for lists above 128), the last block not full
    g = torch.Generator(device="cuda").manual_seed(M)
    z = (3 * torch.randn((M, V + 3), generator=g, device="cuda")).to(DT[dtype][1])[:, :V]
    v, i = lists(g, z, k, ragged=True)
    i[5, 1:] = i[5, 0].clone()  # one class in every slot
    run_distill(z, v, i, 2.0, torch.rand(M, generator=g, device="cuda"))
    run_distill(z, v, i, 1.0, in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_long_lists_with_a_class_named_twice(dtype):
    g = torch.Generator(device="cuda").manual_seed(8)
    for V, k in ((1000, 300), (40000, 1024)):
        z = (3 * torch.randn((3, V), generator=g, device="cuda")).to(DT[dtype][1])
        v, i = lists(g, z, k)
        i[1, 200] = i[1, 3]
        i[2, 100:] = -1
        run_distill(z, v, i, 2.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,k", [(400, 1000, 30), (300, 4099, 64), (297, 8000, 5), (600, 3, 3)])
def test_top_of_many_short_rows(M, V, k, dtype):
    g = torch.Generator(device="cuda").manual_seed(V)
    z = 3 * torch.randn((M, V), generator=g, device="cuda")
    z[3] = 0
    z[4] = torch.arange(V, device="cuda") % 3
    z[5, ::2] = float("nan")
    if z[6:7].element_size() * V <= 16384:
        run_top(z.to(DT[dtype][1]), k)


def test_top_with_many_hot_threads():
    # ascending, descending and blockwise rows: the bound from the threads' maxima is poor or exact
    V = 40000
    a = torch.arange(V, device="cuda").float()
    rows = torch.stack([a, -a, (a // 512) + 1e-3 * (a % 512), a % 512, torch.where(a < 20000, 1.0, 0.0) + 1e-6 * a])
    run_top(rows, 256)
    run_top(rows, 1)
    run_top(rows.to(torch.bfloat16), 100)


@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("M,K,C", [(2600, 2700, 1111), (50176, 70, 64), (12544, 408, 520), (2049, 2560, 129)])
def test_linear_several_tiles_a_block(M, K, C, w_block):
    run_linear(None, M, K, C, K, C, w_block=w_block, y="bf16" if w_block == 1 else "f32", act=2, seed=3)


@pytest.mark.parametrize("M", [3, 100, 2600])
def test_linear_output_that_starts_anywhere(M):
    rng = np.random.default_rng(1)
    K, C = 2600 if M > 1000 else 200, 256
    x, sx, xv, sxv = operand(rng, M, C, "e4m3", 1, 1.0)
    w, sw, wv, swv = operand(rng, K, C, "e4m3", 128, 0.1)
    ref, size = f8_ref.linear(xv, sxv, wv, swv, 128, None, 0, M, K, C)
    for dtype, bf16 in ((torch.bfloat16, True), (torch.float32, False)):
        big = torch.full((M * K + 64,), -7.0, dtype=dtype, device="cuda")
        for shift in (1, 3, 8):
            big.fill_(-7)
            d = sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=K, Cmax=C, w_block_rows=128, y_dtype=sgs.SGS_BF16 if bf16 else sgs.SGS_F32)
            sgs.linear_f8(d, x.data_ptr(), sx.data_ptr(), w.data_ptr(), sw.data_ptr(), 0, big[shift:].data_ptr(), stream())
            got = big.double().cpu().numpy()
            assert (got[:shift] == -7).all() and (got[shift + M * K:] == -7).all()
            err = np.abs(got[shift:shift + M * K].reshape(M, K) - ref)
            assert (err <= f8_ref.linear_tolerance(ref, size, C, 0, bf16)).all()


@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("M,K,C", [(64, 203, 1200), (33, 1000, 8192), (200, 201, 1300), (300, 130, 4100), (129, 1100, 2100), (64, 4700, 1100), (16, 9, 9000)])
def test_linear_reduction_shared_by_a_cluster(M, K, C, w_block):
    # two to eight blocks share it, the last with fewer of its blocks or none to spare; rows of the output that do not start on four elements
    run_linear(None, M, K, C, K, C, w_block=w_block, y="f32", act=2, seed=K)
    run_linear(None, M, K, C, K + 5, C + 40, w_block=w_block, y="bf16", ldy=K + 3, ldsx=M + 1, ldsw=K + 9 if w_block == 1 else 60, seed=C)
    run_linear(None, M, K, C, K, C, w_block=w_block, y="bf16", act=1, bias=False, ldy=(K + 7) // 4 * 4, seed=C)


@pytest.mark.parametrize("M,K,C", [(64, 320, 640), (129, 300, 1024), (600, 1030, 1200), (1100, 4000, 1200), (1290, 4090, 300)])
def test_linear_either_side_of_the_choice_of_form(M, K, C):
    run_linear(None, M, K, C, K, C, y="bf16", act=1, seed=M)
    run_linear(None, M, K, C, K, C, w_block=1, y="f32", seed=M)


def test_offsets_beyond_32_bits():
    # a few rows far apart: element offsets up to 2.4e9
    pitch, M, V = 1 << 28, 10, 3000
    g = torch.Generator(device="cuda").manual_seed(1)
    big = torch.empty((M, pitch), dtype=torch.bfloat16, device="cuda")
    z = big[:, :V]
    z.copy_(3 * torch.randn((M, V), generator=g, device="cuda"))
    run_top(z, 20)
    v, i = lists(g, z, 20)
    run_distill(z, v, i, 2.0)
    d = sgs.DistillDesc(rows=M, classes=V, top=20, dtype=sgs.SGS_BF16, ldz=pitch, lddz=pitch, temperature=2.0, grad_scale=1.0)
    loss = torch.empty(M, device="cuda")
    ref = f8_ref.distill(z.double().cpu().numpy(), v.cpu().numpy(), i.cpu().numpy(), 2.0, np.ones(M))
    q, s, qt, st = quantize(z, "e4m3", 1)
    check_side(q, s, z.double().cpu().numpy(), "e4m3", 1)
    check_side(qt, st, z.double().cpu().numpy().T, "e4m3", 1)
    sgs.distill(d, z.data_ptr(), v.data_ptr(), i.data_ptr(), 0, loss.data_ptr(), 0, z.data_ptr(), stream())  # the gradient in the logits' place
    assert np.abs(z.double().cpu().numpy() - ref[2]).max() <= 2.0 ** -7
    # codes whose rows are far apart, and a layer's output
    codes = torch.empty((M, pitch), dtype=torch.uint8, device="cuda")
    scale = torch.empty((24, M), device="cuda")
    x = torch.randn((M, V), generator=g, device="cuda")
    sgs.quantize_f8(sgs.QuantizeF8Desc(rows=M, cols=V, dtype=sgs.SGS_F32, block_rows=1, ldq=pitch), x.data_ptr(), codes.data_ptr(), scale.data_ptr(), stream=stream())
    want, sc = f8_ref.quantize(x.double().cpu().numpy(), "e4m3", 1)
    np.testing.assert_array_equal(f8_ref.decode(codes[:, :V].cpu().numpy(), "e4m3"), want)
    wq, ws, wv, wsv = operand(np.random.default_rng(2), 200, V, "e4m3", 128, 0.02)
    for M2 in (M, 300):
        y = torch.empty((M2, pitch // 32 if M2 > M else pitch), device="cuda")
        xq, xs, xv, xsv = (codes, scale, want, sc) if M2 == M else operand(np.random.default_rng(3), M2, V, "e4m3", 1, 1.0)
        d = sgs.LinearF8Desc(M=M2, K=200, C=V, Kmax=200, Cmax=V, w_block_rows=128, y_dtype=sgs.SGS_F32, ldx=pitch if M2 == M else 0, ldy=y.stride(0))
        sgs.linear_f8(d, xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), ws.data_ptr(), 0, y.data_ptr(), stream())
        r, size = f8_ref.linear(xv, xsv, wv, wsv, 128, None, 0, M2, 200, V)
        assert (np.abs(y[:, :200].double().cpu().numpy() - r) <= f8_ref.linear_tolerance(r, size, V, 0, False)).all()
        del y


def test_host_threads_with_streams_of_their_own():
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((200, 640), generator=g, device="cuda").to(torch.bfloat16)
    wq, ws, _, _ = quantize(torch.randn((520, 640), generator=g, device="cuda"), "e4m3", 128, sides="row")
    results, errors = [None] * 4, []

    def work(n):
        try:
            st = torch.cuda.Stream()
            q, s = torch.empty((200, 640), dtype=torch.uint8, device="cuda"), torch.empty((5, 200), device="cuda")
            y, v, i = torch.empty((200, 520), device="cuda"), torch.empty((200, 30), device="cuda"), torch.empty((200, 30), dtype=torch.int32, device="cuda")
            torch.cuda.synchronize()
            for _ in range(20):
                sgs.quantize_f8(sgs.QuantizeF8Desc(rows=200, cols=640, dtype=sgs.SGS_BF16, block_rows=1), x.data_ptr(), q.data_ptr(), s.data_ptr(), stream=st.cuda_stream)
                sgs.linear_f8(sgs.LinearF8Desc(M=200, K=520, C=640, Kmax=520, Cmax=640, w_block_rows=128, y_dtype=sgs.SGS_F32), q.data_ptr(), s.data_ptr(),
                              wq.data_ptr(), ws.data_ptr(), 0, y.data_ptr(), st.cuda_stream)
                sgs.top_logits(sgs.TopLogitsDesc(rows=200, classes=520, top=30, dtype=sgs.SGS_F32), y.data_ptr(), v.data_ptr(), i.data_ptr(), st.cuda_stream)
            st.synchronize()
            results[n] = (y, v, i)
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(n,)) for n in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for r in results[1:]:
        for a, b in zip(results[0], r):
            assert torch.equal(a, b)


FIRST_CALL_CAPTURED = """
import torch
import paper_2306_17266_b200 as sgs
x = torch.full((16, 128), 0x38, dtype=torch.uint8, device="cuda")  # ones
s = torch.ones((1, 16), device="cuda")
y = torch.zeros((16, 16), device="cuda")
d = sgs.LinearF8Desc(M=16, K=16, C=128, Kmax=16, Cmax=128, w_block_rows=1, y_dtype=sgs.SGS_F32)
call = lambda st: sgs.linear_f8(d, x.data_ptr(), s.data_ptr(), x.data_ptr(), s.data_ptr(), 0, y.data_ptr(), st.cuda_stream)
st, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=st):
    y.add_(1)
    try:
        call(st)
        raise SystemExit("not refused")
    except sgs.SgsError as e:
        assert e.status == sgs.binding.SGS_EINVAL, e.status
graph.replay()
torch.cuda.synchronize()
assert (y == 1).all()
call(other)
torch.cuda.synchronize()
assert (y == 128).all()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=st):
    call(st)
y.zero_()
graph.replay()
torch.cuda.synchronize()
assert (y == 128).all() and sgs.device_status() == 0
"""


def test_first_layer_call_under_capture_is_refused_and_the_capture_goes_on():
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_CAPTURED], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
