"""8-bit floating point: block quantisation and the sliced linear layer against 64-bit statements of their formulas."""
import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from tests import f8_ref

pytestmark = pytest.mark.gpu

FMT = {"e4m3": sgs.SGS_E4M3, "e5m2": sgs.SGS_E5M2}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
DT = {"bf16": (sgs.SGS_BF16, torch.bfloat16), "f32": (sgs.SGS_F32, torch.float32)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def round16(n):
    return (n + 15) // 16 * 16


def quantize(x, fmt, block, ldq=0, ldqt=0, lds=0, ldst=0, sides="both", fill=0x55):
    """(codes, scales, transposed codes, transposed scales) with everything the call must not touch set to `fill` / -7."""
    R, C = x.shape
    rb, cb = -(-R // 128), -(-C // 128)
    q = torch.full((R, ldq or round16(C)), fill, dtype=torch.uint8, device="cuda")
    qt = torch.full((C, ldqt or round16(R)), fill, dtype=torch.uint8, device="cuda")
    s = torch.full((cb, lds or (R if block == 1 else rb)), -7.0, device="cuda")
    st = torch.full((rb, ldst or (C if block == 1 else cb)), -7.0, device="cuda")
    d = sgs.QuantizeF8Desc(rows=R, cols=C, dtype=sgs.SGS_BF16 if x.dtype == torch.bfloat16 else sgs.SGS_F32, format=FMT[fmt], block_rows=block,
                           ldx=x.stride(0) if R > 1 else 0, ldq=ldq, ldqt=ldqt, lds=lds, ldst=ldst)
    row, col = sides in ("both", "row"), sides in ("both", "col")
    sgs.quantize_f8(d, x.data_ptr(), q.data_ptr() if row else 0, s.data_ptr() if row else 0, qt.data_ptr() if col else 0,
                    st.data_ptr() if col else 0, stream())
    torch.cuda.synchronize()
    return q, s, qt, st


def check_side(q, s, x, fmt, block, fill=0x55):
    R, C = x.shape
    want, scale = f8_ref.quantize(x, fmt, block)
    q, s = q.cpu().numpy(), s.cpu().numpy()
    lines = scale.shape[1]
    np.testing.assert_array_equal(s[:, :lines], scale)
    assert (s[:, lines:] == -7).all()
    np.testing.assert_array_equal(f8_ref.decode(q[:, :C], fmt), want)
    assert (q[:, C:] == fill).all()


SIZES = [(1, 1), (1, 128), (3, 7), (128, 128), (127, 129), (130, 1), (257, 384), (5, 1000), (300, 17), (64, 2056)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("size", SIZES)
def test_quantize_both_sides(size, block, fmt, dtype):
    rng = np.random.default_rng(size[0] * 31 + size[1])
    x = rng.standard_normal(size) * np.exp(2 * rng.standard_normal((size[0], 1)))
    x[rng.random(size) < 0.05] = 0
    t = torch.from_numpy(x).to(DT[dtype][1]).cuda()
    q, s, qt, st = quantize(t, fmt, block)
    v = t.double().cpu().numpy()
    check_side(q, s, v, fmt, block)
    check_side(qt, st, v.T, fmt, block)


@pytest.mark.parametrize("sides", ["row", "col"])
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_pitches_and_unaligned_rows(block, sides):
    # rows of x that start anywhere, odd pitches everywhere, one side alone
    big = torch.randn((150, 260), device="cuda").to(torch.bfloat16)
    x = big[3:146, 5:206]
    q, s, qt, st = quantize(x, "e4m3", block, ldq=203, ldqt=149, lds=151, ldst=211, sides=sides)
    v = x.double().cpu().numpy()
    if sides == "row":
        check_side(q, s, v, "e4m3", block)
        assert (qt == 0x55).all() and (st == -7).all()
    else:
        check_side(qt, st, v.T, "e4m3", block)
        assert (q == 0x55).all() and (s == -7).all()


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
def test_quantize_extremes(block, fmt):
    # zeros, the least and largest magnitudes, ties, NaN and infinities next to ordinary values
    x = np.zeros((140, 300), dtype=np.float32)
    rng = np.random.default_rng(5)
    x[1] = np.float32(3.4028235e38) * rng.uniform(-1, 1, 300).astype(np.float32)
    x[2] = 1e-45
    x[3] = 2.0 ** -126 * rng.integers(-9, 9, 300)
    x[4, ::7] = np.nan
    x[5, :128] = np.inf
    x[6] = rng.standard_normal(300)
    x[6, 5], x[6, 200] = -np.inf, np.nan
    x[7] = np.arange(300) * 2.0 ** -4
    x[8], x[9] = f8_ref.FMAX[fmt], np.nextafter(np.float32(f8_ref.FMAX[fmt]), np.float32(1e9))
    x[129:] = rng.standard_normal((11, 300))
    q, s, qt, st = quantize(torch.from_numpy(x).cuda(), fmt, block)
    check_side(q, s, x, fmt, block)
    check_side(qt, st, x.T, fmt, block)


def operand(rng, rows, cols, fmt, block, spread, pitch=0, line=0, general=False):
    """Codes and scales on the device, their values and scales on the host.  general: scales that are no powers of two."""
    v, s = f8_ref.quantize(rng.standard_normal((rows, cols)) * spread * np.exp(0.5 * rng.standard_normal((rows, 1))), fmt, block)
    if general:
        s = s * rng.uniform(0.5, 1.0, s.shape)
    s = s.astype(np.float32)
    ld = pitch or round16(cols)
    codes = torch.full((rows, ld), 0x7F, dtype=torch.uint8, device="cuda")  # NaN wherever nothing may be read
    codes[:, :cols] = torch.from_numpy(v).to(torch.float32).to(F8[fmt]).view(torch.uint8).cuda()
    scales = torch.full((s.shape[0], line or s.shape[1]), float("nan"), device="cuda")
    scales[:, :s.shape[1]] = torch.from_numpy(s).cuda()
    return codes, scales, v, s


def run_linear(c, M, K, C, Kmax, Cmax, xf="e4m3", wf="e4m3", w_block=128, y="bf16", act=0, bias=True, ldx=0, ldw=0, ldy=0, ldsx=0, ldsw=0, seed=0):
    rng = np.random.default_rng(seed)
    x, sx, xv, sxv = operand(rng, M, C, xf, 1, 1.0, ldx, ldsx, general=True)
    w, sw, wv, swv = operand(rng, Kmax, Cmax, wf, w_block, np.sqrt(2.0 / C), ldw, ldsw, general=True)
    b = rng.standard_normal(Kmax).astype(np.float32) * 0.1 if bias else None
    db = torch.from_numpy(b).cuda() if bias else None
    out = torch.full((M + 1, ldy or K), -77.0, dtype=DT[y][1], device="cuda")
    d = sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=Kmax, Cmax=Cmax, x_format=FMT[xf], w_format=FMT[wf], w_block_rows=w_block, y_dtype=DT[y][0], act=act,
                         ldx=ldx, ldw=ldw, ldy=ldy, ldsx=ldsx, ldsw=ldsw)
    for _ in range(2):
        sgs.linear_f8(d, x.data_ptr(), sx.data_ptr(), w.data_ptr(), sw.data_ptr(), db.data_ptr() if bias else 0, out.data_ptr(), stream())
    torch.cuda.synchronize()
    assert sgs.device_status() == 0
    ref, size = f8_ref.linear(xv, sxv, wv, swv, w_block, b, act, M, K, C)
    got = out.double().cpu().numpy()
    err = np.abs(got[:M, :K] - ref)
    tol = f8_ref.linear_tolerance(ref, size, C, act, y == "bf16")
    assert np.isfinite(got[:M, :K]).all()
    assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
    assert (got[M:] == -77).all() and (got[:, K:] == -77).all()  # what lies beyond the output is left as it was


LINEAR = [
    # M, K, C, Kmax, Cmax
    (1, 8, 16, 8, 16), (1, 1, 1, 1, 1), (1, 1000, 2048, 1000, 2048), (2, 129, 130, 300, 300), (7, 64, 128, 64, 128), (16, 1000, 512, 1000, 512),
    (17, 200, 100, 256, 384), (33, 1000, 1000, 1024, 1024), (64, 100, 129, 128, 256), (65, 264, 1040, 300, 1100), (100, 257, 640, 512, 640),
    (128, 128, 256, 128, 256), (129, 408, 512, 512, 512), (200, 13, 4096, 13, 4096), (640, 520, 300, 520, 300), (1000, 1000, 200, 1000, 200),
    (4096, 300, 96, 300, 96), (300, 4100, 64, 4100, 64), (2500, 2500, 260, 2500, 260),
]


@pytest.mark.parametrize("w_block", [1, 128])
@pytest.mark.parametrize("case", LINEAR)
def test_linear_sizes(case, w_block):
    M, K, C, Kmax, Cmax = case
    run_linear(None, M, K, C, Kmax, Cmax, w_block=w_block, y="f32", seed=M + K)
    run_linear(None, M, K, C, Kmax, Cmax, w_block=w_block, y="bf16", act=1 + (M & 1), bias=bool(K & 1), seed=M + C)


@pytest.mark.parametrize("formats", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("M", [3, 40, 300])
def test_linear_formats(M, formats):
    run_linear(None, M, 200, 500, 200, 500, *formats, y="f32", seed=M)


@pytest.mark.parametrize("M", [1, 20, 150])
@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("w_block", [1, 128])
def test_linear_pitches(M, y, w_block):
    run_linear(None, M, 203, 333, 260, 400, y=y, w_block=w_block, ldx=352, ldw=416, ldy=207, ldsx=M + 3, ldsw=301, seed=M)
    run_linear(None, M, 201, 333, 260, 400, y=y, w_block=w_block, ldx=336, ldw=400, ldy=208, ldsx=M, ldsw=0, act=2, seed=M)


def test_linear_nan_stays_in_its_row():
    x = torch.randn((130, 256), device="cuda")
    x[77, 200] = float("nan")
    q, s, _, _ = quantize(x, "e4m3", 1, sides="row")
    wq, ws, _, _ = quantize(torch.randn((300, 256), device="cuda"), "e4m3", 128, sides="row")
    for M in (130, 78):
        y = torch.zeros((M, 300), device="cuda")
        d = sgs.LinearF8Desc(M=M, K=300, C=256, Kmax=300, Cmax=256, w_block_rows=128, y_dtype=sgs.SGS_F32, ldsx=130)
        sgs.linear_f8(d, q.data_ptr(), s.data_ptr(), wq.data_ptr(), ws.data_ptr(), 0, y.data_ptr(), stream())
        nan = torch.isnan(y).cpu().numpy()
        assert nan[77].all() and nan.sum() == 300


def test_gradients_of_a_layer():
    # y = x w^T, loss = sum(g * y): dx = g w and dw = g^T x from the same two calls, against the formulas on the decoded operands and
    # against differences of the 64-bit loss
    M, K, C = 75, 130, 200
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w, g = (torch.randn(s, generator=gen, device="cuda") for s in ((M, C), (K, C), (M, K)))
    xq, xs, xqt, xst = quantize(x, "e4m3", 1)
    wq, ws, wqt, wst = quantize(w, "e4m3", 128)
    gq, gs, gqt, gst = quantize(g, "e5m2", 1)
    dx, dw = torch.zeros((M, C), device="cuda"), torch.zeros((K, C), device="cuda")
    sgs.linear_f8(sgs.LinearF8Desc(M=M, K=C, C=K, Kmax=C, Cmax=K, x_format=sgs.SGS_E5M2, w_block_rows=128, y_dtype=sgs.SGS_F32),
                  gq.data_ptr(), gs.data_ptr(), wqt.data_ptr(), wst.data_ptr(), 0, dx.data_ptr(), stream())
    sgs.linear_f8(sgs.LinearF8Desc(M=K, K=C, C=M, Kmax=C, Cmax=M, x_format=sgs.SGS_E5M2, w_block_rows=1, y_dtype=sgs.SGS_F32),
                  gqt.data_ptr(), gst.data_ptr(), xqt.data_ptr(), xst.data_ptr(), 0, dw.data_ptr(), stream())
    torch.cuda.synchronize()

    def values(q, s, shape, fmt, block):
        R, Cc = shape
        return f8_ref.decode(q.cpu().numpy()[:, :Cc], fmt) * np.repeat(np.repeat(s.double().cpu().numpy().T, block, 0)[:R], 128, 1)[:, :Cc]
    G, W = values(gq, gs, (M, K), "e5m2", 1), values(wqt, wst, (C, K), "e4m3", 128).T
    np.testing.assert_array_equal(W, values(wq, ws, (K, C), "e4m3", 128))  # square blocks: the transpose has the same values
    Gt, Xt = values(gqt, gst, (K, M), "e5m2", 1).T, values(xqt, xst, (C, M), "e4m3", 1).T
    for got, ref, size, n in ((dx, G @ W, np.abs(G) @ np.abs(W), K), (dw, Gt.T @ Xt, np.abs(Gt).T @ np.abs(Xt), M)):
        err = np.abs(got.double().cpu().numpy() - ref)
        assert (err <= f8_ref.linear_tolerance(ref, size, n, 0, False)).all()
    # differences: the loss is linear in x and in w, so a step of 1 gives the derivative but for the sums' rounding
    loss = lambda X, Wm, Gm: float(np.sum(Gm * (X @ Wm.T)))  # noqa: E731
    X = values(xq, xs, (M, C), "e4m3", 1)
    for i, j in ((0, 0), (74, 199), (40, 100)):
        X2 = X.copy(); X2[i, j] += 1
        assert abs(float(dx[i, j]) - (loss(X2, W, G) - loss(X, W, G))) <= 1e-4 * (1 + np.abs(G[i]) @ np.abs(W[:, j]))
    for i, j in ((0, 0), (129, 199), (60, 3)):
        W2 = W.copy(); W2[i, j] += 1
        assert abs(float(dw[i, j]) - (loss(Xt, W2, Gt) - loss(Xt, W, Gt))) <= 1e-4 * (1 + np.abs(Gt[:, i]) @ np.abs(Xt[:, j]))


def test_calls_are_refused_and_write_nothing():
    x = torch.zeros((16, 32), dtype=torch.uint8, device="cuda")
    s = torch.ones((1, 16), device="cuda")
    y = torch.full((16, 16), 7.0, device="cuda")
    ok = dict(M=16, K=16, C=32, Kmax=16, Cmax=32, w_block_rows=1, y_dtype=sgs.SGS_F32)

    def call(status, xp=None, yp=None, **change):
        with pytest.raises(sgs.SgsError) as e:
            sgs.linear_f8(sgs.LinearF8Desc(**{**ok, **change}), xp or x.data_ptr(), s.data_ptr(), x.data_ptr(), s.data_ptr(), 0, yp or y.data_ptr(), stream())
        assert e.value.status == status
    call(sgs.binding.SGS_EUNSUPPORTED, xp=x.data_ptr() + 8)
    call(sgs.binding.SGS_EUNSUPPORTED, ldx=40)
    call(sgs.binding.SGS_EINVAL, ldx=16)
    call(sgs.binding.SGS_EINVAL, K=17)
    call(sgs.binding.SGS_EINVAL, w_block_rows=64)
    host = torch.zeros(4096)
    call(sgs.binding.SGS_EINVAL, yp=host.data_ptr())  # plain host memory
    with pytest.raises(sgs.SgsError) as e:
        sgs.quantize_f8(sgs.QuantizeF8Desc(rows=4, cols=4, dtype=sgs.SGS_F32, block_rows=1), host.data_ptr(), x.data_ptr(), s.data_ptr(), 0, 0, stream())
    assert e.value.status == sgs.binding.SGS_EINVAL
    torch.cuda.synchronize()
    assert (y == 7).all()
