"""Top logits and the distillation loss with its gradient against 64-bit statements of their formulas."""
import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests import f8_ref

pytestmark = pytest.mark.gpu

DT = {"bf16": (sgs.SGS_BF16, torch.bfloat16), "f32": (sgs.SGS_F32, torch.float32)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def run_top(z, k, ldt=0):
    M, V = z.shape
    values = torch.full((M + 1, ldt or k), -7.0, device="cuda")
    index = torch.full((M + 1, ldt or k), -7, dtype=torch.int32, device="cuda")
    d = sgs.TopLogitsDesc(rows=M, classes=V, top=k, dtype=sgs.SGS_BF16 if z.dtype == torch.bfloat16 else sgs.SGS_F32, ldz=z.stride(0) if M > 1 else 0, ldt=ldt)
    sgs.top_logits(d, z.data_ptr(), values.data_ptr(), index.data_ptr(), stream())
    torch.cuda.synchronize()
    v = z.double().cpu().numpy()
    want = f8_ref.top(v, k)
    got = index.cpu().numpy()
    np.testing.assert_array_equal(got[:M, :k], want)
    np.testing.assert_array_equal(values.double().cpu().numpy()[:M, :k], np.take_along_axis(v, want, 1))
    assert (got[M:] == -7).all() and (got[:, k:] == -7).all() and (values[M:] == -7).all() and (values[:, k:] == -7).all()


TOP = [(1, 1, 1), (3, 2, 2), (5, 33, 7), (64, 1000, 32), (2, 1000, 256), (3, 256, 256), (1, 1024, 1), (2, 1025, 256), (4, 5000, 64), (3, 32771, 100),
       (1, 131072, 128), (2, 200003, 256), (200, 4099, 17), (1, 1000003, 50)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", TOP)
def test_top_of_random_rows(case, dtype):
    M, V, k = case
    g = torch.Generator(device="cuda").manual_seed(V + k)
    run_top((3 * torch.randn((M, V), generator=g, device="cuda")).to(DT[dtype][1]), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(40, 40), (1000, 10), (3000, 200), (70001, 256)])
def test_top_of_rows_with_many_equal_values(V, k, dtype):
    rows = [torch.zeros(V), -torch.zeros(V), torch.full((V,), float("-inf")), torch.arange(V).float(), -torch.arange(V).float(), torch.arange(V).float() % 2,
            torch.full((V,), float("nan")), torch.full((V,), torch.finfo(torch.bfloat16).min)]
    mixed = torch.zeros(V)
    mixed[1::2] = -0.0
    mixed[V // 2] = 1.0
    odd = torch.randn(V)
    odd[::3], odd[1], odd[V - 1], odd[V // 2] = float("-inf"), float("inf"), float("nan"), -float("nan")
    almost = torch.full((V,), -1.0)
    almost[V - 1] = -2.0
    run_top(torch.stack(rows + [mixed, odd, almost]).to(DT[dtype][1]).cuda(), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_top_of_rows_at_odd_addresses(dtype):
    big = torch.randn((9, 5003), device="cuda").to(DT[dtype][1])
    run_top(big[1:8, 3:4900], 20, ldt=23)
    run_top(big[1:8, 1:1000], 20, ldt=23)


def run_distill(z, teacher, index, T, row_scale=None, grad_scale=1.0, lddz=0, in_place=False):
    """Loss alone, loss with gradient, and the backward pass from the statistics: all against 64 bits, and the two gradients against each other."""
    M, V = z.shape
    k = index.shape[1]
    bf16 = z.dtype == torch.bfloat16
    ldz = z.stride(0) if M > 1 else V
    if in_place:
        lddz = ldz
    d = sgs.DistillDesc(rows=M, classes=V, top=k, dtype=sgs.SGS_BF16 if bf16 else sgs.SGS_F32, ldz=ldz, lddz=lddz, ldt=k, temperature=T, grad_scale=grad_scale)
    zh = z.double().cpu().numpy()
    th, ih = teacher.cpu().numpy(), index.cpu().numpy()
    rs = row_scale.cpu().numpy().astype(np.float64) if row_scale is not None else np.ones(M)
    coef = np.float64(np.float32(grad_scale)) * rs
    loss, stat, dz, Q, P = f8_ref.distill(zh, th, ih, T, coef)
    tol = f8_ref.distill_tolerance(zh, th, ih, T)
    rsp = row_scale.data_ptr() if row_scale is not None else 0
    outs = []
    for mode in ("loss", "step", "backward"):
        gl = torch.full((M + 1,), -7.0, device="cuda")
        gs = torch.full((M + 1, 2), -7.0, device="cuda")
        src = z
        if in_place and mode != "loss":
            src = torch.empty((M, ldz), dtype=z.dtype, device="cuda")[:, :V]
            src.copy_(z)
            out = src
        else:
            out = torch.full((M + 1, lddz or V), -7.0, dtype=z.dtype, device="cuda")
        if mode == "backward":
            sgs.distill_backward(d, src.data_ptr(), teacher.data_ptr(), index.data_ptr(), kept.data_ptr(), rsp, out.data_ptr(), stream())
        else:
            sgs.distill(d, src.data_ptr(), teacher.data_ptr(), index.data_ptr(), rsp, gl.data_ptr(), gs.data_ptr(), out.data_ptr() if mode == "step" else 0, stream())
        torch.cuda.synchronize()
        if mode != "backward":
            kept = gs
            l = gl.double().cpu().numpy()
            assert l[M] == -7 and (gs[M] == -7).all()
            fine = np.abs(loss) <= 3.4028235e38  # (a value beyond fp32 is infinite there: a mask of the type's lowest value, named by the teacher)
            np.testing.assert_array_equal(l[:M][~fine], np.where(np.isfinite(loss), np.inf, loss)[~fine])
            size = T * T * tol * (1 + np.abs(np.where(fine, loss, 0)) / (T * T))
            assert (np.abs(l[:M] - loss)[fine] <= size[fine]).all(), (l[:M], loss)
            st = gs.double().cpu().numpy()[:M]
            np.testing.assert_array_equal(st[:, 0], stat[:, 0])
            fine = np.isfinite(stat[:, 1])
            np.testing.assert_array_equal(st[~fine, 1], stat[~fine, 1])
            assert (np.abs(st[fine, 1] - stat[fine, 1]) <= 2.0 ** -24 * (64 + V / 256) * (1 + np.abs(stat[fine, 1]))).all()
        if mode != "loss":
            got = out.double().cpu().numpy()
            if not in_place:
                assert (got[M:] == -7).all() and (got[:, V:] == -7).all()
            got = got[:M, :V]
            # an exponent of the size of the row's spread may be in use at any class: its roundings count relative to q
            spread = np.where(np.isfinite(zh), zh.max(1, keepdims=True) - zh, 0) / T
            rel = tol[:, None] + 2.0 ** -24 * 8 * np.nan_to_num(spread, posinf=0)
            bound = np.abs(coef)[:, None] * T * (Q + P) * rel + 1e-37
            if bf16:
                bound = bound + 2.0 ** -8 * (np.abs(dz) + bound)
            err = np.abs(got - dz)
            assert (err <= bound).all(), (mode, float((err / bound).max()), np.unravel_index((err / bound).argmax(), err.shape))
            outs.append(got)
    return outs


def lists(g, z, k, ragged=False):
    t = z.float() + 1.5 * torch.randn(z.shape, generator=g, device="cuda")
    t[torch.isinf(z)] = -1e4
    v, i = torch.topk(t, k, dim=1)
    i = i.to(torch.int32)
    if ragged:
        n = torch.randint(0, k + 1, (z.shape[0], 1), generator=g, device="cuda")
        n[0] = 0
        i[torch.arange(k, device="cuda")[None] >= n] = -1
    return v.contiguous(), i.contiguous()


DISTILL = [(1, 1, 1), (1, 2, 1), (3, 7, 7), (64, 1000, 32), (5, 1000, 1000), (2, 1024, 1024), (4, 4096, 64), (3, 10007, 100), (2, 65536, 128), (1, 100003, 17),
           (1, 131072, 64), (300, 515, 20), (2, 250008, 200), (1, 600001, 8)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", DISTILL)
def test_distill(case, dtype):
    M, V, k = case
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (3 * torch.randn((M, V), generator=g, device="cuda")).to(DT[dtype][1])
    v, i = lists(g, z, k, ragged=M > 1)
    run_distill(z, v, i, 2.0, torch.rand(M, generator=g, device="cuda"), 0.5)


@pytest.mark.parametrize("T", [0.25, 1.0, 4.0])
@pytest.mark.parametrize("V", [777, 20000])
def test_distill_temperatures_pitches_and_in_place(V, T):
    g = torch.Generator(device="cuda").manual_seed(7)
    for dtype in ("bf16", "f32"):
        for pad in (0, 3, 8):
            z = (4 * torch.randn((5, V + pad), generator=g, device="cuda")).to(DT[dtype][1])[:, :V]
            v, i = lists(g, z, 30, ragged=True)
            run_distill(z, v, i, T, lddz=V + 5)
            run_distill(z, v, i, T, in_place=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [600, 30000])
def test_distill_masks_and_lists(V, dtype):
    g = torch.Generator(device="cuda").manual_seed(9)
    low = torch.finfo(DT[dtype][1]).min
    z = 3 * torch.randn((9, V), generator=g, device="cuda")
    v, i = lists(g, z, 40)
    z[0, V // 3:] = float("-inf")        # masked classes, some of them named: an infinite loss
    z[1] = float("-inf")                 # nothing left
    z[2, 5:] = low                       # masks of the type's lowest value
    z[3] = low                           # a row of it
    z[4, 7] = 1e5                        # one class alone
    i[5, ::2] = V                        # outside
    i[5, 1] = -5
    i[6, 1:] = i[6, 0]                   # the same class in every slot
    v[7, 3:] = float("-inf")             # a teacher's own masks
    v[8] = float("-inf")                 # nothing named
    i[0, 10:] = torch.arange(30, device="cuda", dtype=torch.int32)
    run_distill(z.to(DT[dtype][1]), v, i, 2.0)


@pytest.mark.parametrize("V", [600, 30000])
def test_distill_nan_and_rows_that_do_not_count(V):
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn((4, V), generator=g, device="cuda")
    v, i = lists(g, z, 8)
    z[0, 3] = float("nan")
    z[1, 3] = float("nan")
    i[1] = -1                            # no list: loss and gradient 0 whatever the logits
    z[2, 3] = float("nan")
    scale = torch.tensor([1.0, 1.0, 0.0, 1.0], device="cuda")
    loss, stat, dz = torch.empty(4, device="cuda"), torch.empty((4, 2), device="cuda"), torch.empty((4, V), device="cuda")
    d = sgs.DistillDesc(rows=4, classes=V, top=8, dtype=sgs.SGS_F32, temperature=1.0, grad_scale=1.0)
    for mode in ("step", "backward"):
        dz.fill_(5)
        if mode == "step":
            sgs.distill(d, z.data_ptr(), v.data_ptr(), i.data_ptr(), scale.data_ptr(), loss.data_ptr(), stat.data_ptr(), dz.data_ptr(), stream())
        else:
            sgs.distill_backward(d, z.data_ptr(), v.data_ptr(), i.data_ptr(), stat.data_ptr(), scale.data_ptr(), dz.data_ptr(), stream())
        torch.cuda.synchronize()
        assert torch.isnan(loss[0]) and loss[1] == 0 and torch.isnan(loss[2]) and torch.isfinite(loss[3])
        assert torch.isnan(dz[0]).all() and (dz[1] == 0).all() and (dz[2] == 0).all() and torch.isfinite(dz[3]).all()


def test_gradient_against_differences():
    g = torch.Generator(device="cuda").manual_seed(4)
    z = 2 * torch.randn((3, 50), generator=g, device="cuda")
    v, i = lists(g, z, 12)
    i[2, 5:] = -1
    i[1, 3] = i[1, 4]
    T = 2.0
    dz = run_distill(z, v, i, T)[0]
    zh, th, ih = z.double().cpu().numpy(), v.cpu().numpy(), i.cpu().numpy()
    h = 1e-4
    for r in range(3):
        for c in list(range(0, 50, 7)) + list(ih[r, :5].clip(0)):
            up, down = zh.copy(), zh.copy()
            up[r, c] += h
            down[r, c] -= h
            slope = (f8_ref.distill(up, th, ih, T, np.ones(3))[0][r] - f8_ref.distill(down, th, ih, T, np.ones(3))[0][r]) / (2 * h)
            assert abs(dz[r, c] - slope) <= 1e-5  # (third derivatives are below T^2 / T^3: h^2 of it; fp32 rounding of the gradient)


def test_logit_calls_are_refused_and_write_nothing():
    z = torch.randn((4, 300), device="cuda")
    v = torch.full((4, 300), 7.0, device="cuda")
    i = torch.full((4, 300), 7, dtype=torch.int32, device="cuda")
    E = sgs.binding.SGS_EINVAL

    def top(zp=None, **change):
        with pytest.raises(sgs.SgsError) as e:
            sgs.top_logits(sgs.TopLogitsDesc(**{**dict(rows=4, classes=300, top=5, dtype=sgs.SGS_F32), **change}), zp or z.data_ptr(), v.data_ptr(), i.data_ptr(), stream())
        assert e.value.status == E
    top(top=301), top(top=257), top(top=0), top(rows=0), top(ldz=299), top(ldt=4), top(dtype=5), top(zp=torch.zeros(1200).data_ptr())

    def dis(zp=None, dz=0, **change):
        ok = dict(rows=4, classes=300, top=5, dtype=sgs.SGS_F32, temperature=1.0, grad_scale=1.0)
        with pytest.raises(sgs.SgsError) as e:
            sgs.distill(sgs.DistillDesc(**{**ok, **change}), zp or z.data_ptr(), z.data_ptr(), i.data_ptr(), 0, v.data_ptr(), 0, dz, stream())
        assert e.value.status == E
    dis(temperature=0.0), dis(temperature=float("nan")), dis(temperature=float("inf")), dis(temperature=-1.0), dis(temperature=1e-45), dis(grad_scale=float("inf"))
    dis(top=0), dis(top=1025, classes=2000, ldz=2000), dis(ldz=5), dis(ldt=4), dis(zp=z.data_ptr() + 2), dis(zp=torch.zeros(1200).data_ptr())
    dis(dz=z.data_ptr(), lddz=301)
    torch.cuda.synchronize()
    assert (v == 7).all() and (i == 7).all()


@pytest.mark.parametrize("V", [500, 40000])
def test_captured_calls_and_another_stream(V):
    # captured at once (no first call outside), replayed on new logits, on a stream of its own
    g = torch.Generator(device="cuda").manual_seed(1)
    M, k = 6, 20
    z = torch.randn((M, V), generator=g, device="cuda")
    values, index = torch.zeros((M, k), device="cuda"), torch.zeros((M, k), dtype=torch.int32, device="cuda")
    loss, dz = torch.zeros(M, device="cuda"), torch.zeros((M, V), device="cuda")
    student = torch.randn((M, V), generator=g, device="cuda")
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        sgs.top_logits(sgs.TopLogitsDesc(rows=M, classes=V, top=k, dtype=sgs.SGS_F32), z.data_ptr(), values.data_ptr(), index.data_ptr(), st.cuda_stream)
        sgs.distill(sgs.DistillDesc(rows=M, classes=V, top=k, dtype=sgs.SGS_F32, temperature=1.0, grad_scale=1.0), student.data_ptr(), values.data_ptr(),
                    index.data_ptr(), 0, loss.data_ptr(), 0, dz.data_ptr(), st.cuda_stream)
    for seed in (5, 6):
        z.copy_(torch.randn((M, V), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        student.copy_(z + 0.5)  # the same distribution up to the lists
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        st.synchronize()
        zh = z.double().cpu().numpy()
        np.testing.assert_array_equal(index.cpu().numpy(), f8_ref.top(zh, k))
        sh = student.double().cpu().numpy()
        ref, _, dref, _, _ = f8_ref.distill(sh, values.cpu().numpy(), index.cpu().numpy(), 1.0, np.ones(M))
        tol = f8_ref.distill_tolerance(sh, values.cpu().numpy(), index.cpu().numpy(), 1.0)
        assert (np.abs(loss.double().cpu().numpy() - ref) <= tol * (1 + np.abs(ref))).all()
        assert np.abs(dz.double().cpu().numpy() - dref).max() <= tol.max()
