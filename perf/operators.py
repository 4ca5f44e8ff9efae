"""Operators on 8-bit floating point layers and on logits, and how they are measured.

``listed()`` names the fixed cases, ``draw(rng)`` gives another of the same ranges, ``prepare`` makes what a program has in
hand before the call, ``run`` is one pass: the plain form in elementary torch operations, or (``own``) the library's call.

Kinds of a case:
  quantize  a matrix in 8-bit floating point with a power-of-two scale per block of 1x128 or 128x128: its codes, those of its
            transpose, or both                      (rows, cols, dtype, format, block, rowwise, transposed)
  linear    y = act(x w^T + bias), x and w in 8 bits with a scale per 128 of the reduction; the first K rows and C columns of
            stored weights                          (M, K, C, Kmax, Cmax, x_format, w_format, w_block, y_dtype, act, bias)
  top       the k largest logits of every row and where they are            (M, V, k, dtype)
  distill   the distillation loss of every row against a teacher's top logits; mode "loss", "step" (loss and gradient) or
            "backward" (gradient from kept statistics)      (M, V, ld, k, dtype, temperature, mode, ragged, padded)
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP_EXPONENT = {"e4m3": 8, "e5m2": 15}  # the largest code is 1.75 * 2^this
ACTS = {"none": 0, "relu": 1, "hswish": 2}


def quantize(rows, cols, dtype, format, block, rowwise, transposed):
    return {"kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "format": format, "block": block, "rowwise": rowwise,
            "transposed": transposed}


def linear(M, K, C, y_dtype, act="none", bias=True, Kmax=0, Cmax=0, x_format="e4m3", w_format="e4m3", w_block=128):
    return {"kind": "linear", "M": M, "K": K, "C": C, "Kmax": Kmax or K, "Cmax": Cmax or C, "x_format": x_format, "w_format": w_format,
            "w_block": w_block, "y_dtype": y_dtype, "act": act, "bias": bias}


def top(M, V, k, dtype):
    return {"kind": "top", "M": M, "V": V, "k": k, "dtype": dtype}


def distill(M, V, k, dtype, mode, temperature, ld=0, ragged=False, padded=0):
    return {"kind": "distill", "M": M, "V": V, "ld": ld or V, "k": k, "dtype": dtype, "temperature": temperature, "mode": mode,
            "ragged": ragged, "padded": padded}


def listed():
    return [
        # activations of 16 maps of 56x56 pixels in front of a pointwise layer
        dict(quantize(50176, 256, "bf16", "e4m3", 1, True, False), name="quantize_activations"),
        # a gradient for both products of a backward pass: rows for the input's, columns for the weights'
        dict(quantize(8192, 8192, "bf16", "e5m2", 1, True, True), name="quantize_gradient"),
        # one token through a wide layer: the weights' bytes are all it costs
        dict(linear(1, 8192, 4096, "bf16", "none", False), name="linear_token"),
        # the classifier of the ResNet-shaped family on 16 images
        dict(linear(16, 1000, 2048, "f32"), name="linear_classifier"),
        # a pointwise layer of that family's SubNets on 16 maps of 28x28: slices of the stored weights, ReLU
        dict(linear(12544, 408, 512, "bf16", "relu", True, 512, 512), name="linear_pointwise"),
        # throughput: a large layer on many tokens
        dict(linear(8192, 8192, 8192, "bf16"), name="linear_large"),
        # gradient of a layer's weights over an odd number of tokens: both sides in blocks of one row, full precision out
        dict(linear(4096, 2048, 8197, "f32", "none", False, x_format="e5m2", w_block=1), name="linear_weight_gradient"),
        # a teacher's top logits: the framework's 1000 classes, and a large odd number of them
        dict(top(64, 1000, 32, "f32"), name="top_classes"),
        dict(top(512, 131071, 64, "bf16"), name="top_vocabulary"),
        # the loss alone, on 64 images of 1000 classes: latency
        dict(distill(64, 1000, 32, "f32", "loss", 4.0), name="distill_classes"),
        # a training step's loss with its gradient; lists of unequal length, rows without any
        dict(distill(2048, 65536, 64, "bf16", "step", 2.0, ragged=True), name="distill_step"),
        # the gradient by itself, rows padded to a multiple of 8 with classes that do not exist
        dict(distill(1000, 100008, 128, "bf16", "backward", 1.0, padded=5), name="distill_backward"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("quantize", "linear", "linear", "top", "distill"))
    if kind == "quantize":
        rows, cols = _log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 8192)
        side = rng.choice(((True, False), (False, True), (True, True)))
        return quantize(rows, cols, rng.choice(("bf16", "f32")), rng.choice(("e4m3", "e5m2")), rng.choice((1, 128)), *side)
    if kind == "linear":
        M, K, C = _log_uniform(rng, 1, 8192), _log_uniform(rng, 8, 8192), _log_uniform(rng, 16, 8192)
        return linear(M, K, C, rng.choice(("bf16", "f32")), rng.choice(("none", "relu", "hswish")), rng.random() < 0.5,
                      K + rng.choice((0, 0, rng.randint(1, 300))), C + rng.choice((0, 0, rng.randint(1, 300))),
                      rng.choice(("e4m3", "e5m2")), rng.choice(("e4m3", "e4m3", "e5m2")), rng.choice((1, 128)))
    V = _log_uniform(rng, 2, 131072)
    M = _log_uniform(rng, 1, min(4096, 2 ** 26 // V))
    k, dtype = rng.randint(1, min(V, 128)), rng.choice(("bf16", "f32"))
    if kind == "top":
        return top(M, V, k, dtype)
    padded = rng.choice((0, 0, min(7, V - 1)))
    return distill(M, V, min(k, V - padded), dtype, rng.choice(("loss", "step", "backward")), rng.choice((1.0, 2.0, 4.0)),
                   V + rng.choice((0, 0, 3, 8)), rng.random() < 0.5, padded)


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _blocks(n):
    return (n + 127) // 128


def _round16(n):
    return (n + 15) // 16 * 16


def _scales(amax, format):
    """Power-of-two scales: the least with which the largest finite value of a block fits the format, 2^-126 at least."""
    mantissa, exponent = torch.frexp(amax)  # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 1 - TOP_EXPONENT[format] + (mantissa > 0.875).to(exponent.dtype)
    e = torch.where(amax > 0, e, torch.full_like(e, -126)).clamp(min=-126)
    return torch.ldexp(torch.ones_like(amax), e)


def _quantized(x, format, block):
    """Codes [R][C] and scales [blocks of columns][rows or blocks of rows] of x, 32-bit arithmetic."""
    R, C = x.shape
    rb = R if block == 1 else _blocks(R)
    v = torch.zeros((rb * block, _blocks(C) * 128), dtype=torch.float32, device=x.device)
    v[:R, :C] = x.float()
    v = v.view(rb, block, _blocks(C), 128)
    magnitude = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v))
    scale = _scales(magnitude.amax((1, 3)), format)
    q = torch.where(torch.isfinite(v), v / scale[:, None, :, None], torch.full_like(v, float("nan"))).to(F8[format])
    return q.view(rb * block, _blocks(C) * 128)[:R, :C], scale.t().contiguous()


def _operand(g, rows, cols, used, format, block, spread):
    """An 8-bit operand as a program keeps it: codes at a pitch of 16 bytes, and scales."""
    x = torch.randn((rows, cols), generator=g, device="cuda") * spread
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=g, device="cuda"))
    q, scale = _quantized(x, format, block)
    codes = torch.zeros((rows, _round16(cols)), dtype=torch.uint8, device="cuda")
    codes[:, :cols] = q.contiguous().view(torch.uint8)
    return codes, scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + 17)
    kind = case["kind"]
    s = {"case": case}
    if kind == "quantize":
        x = torch.randn((case["rows"], case["cols"]), generator=g, device="cuda")
        x *= torch.exp(torch.randn((case["rows"], 1), generator=g, device="cuda"))  # rows of unequal size, as tokens are
        s["x"] = x.to(DTYPE[case["dtype"]])
    elif kind == "linear":
        M, K, C, Kmax, Cmax = (case[n] for n in ("M", "K", "C", "Kmax", "Cmax"))
        s["x"], s["sx"] = _operand(g, M, C, C, case["x_format"], 1, 1.0)
        s["w"], s["sw"] = _operand(g, Kmax, Cmax, C, case["w_format"], case["w_block"], math.sqrt(2.0 / C))
        s["bias"] = 0.1 * torch.randn(Kmax, generator=g, device="cuda") if case["bias"] else None
    elif kind == "top":
        s["z"] = (3.0 * torch.randn((case["M"], case["V"]), generator=g, device="cuda")).to(DTYPE[case["dtype"]])
    else:
        M, V, k, T = case["M"], case["V"], case["k"], case["temperature"]
        z = 3.0 * torch.randn((M, case["ld"]), generator=g, device="cuda")
        teacher = z[:, :V - case["padded"]] + 1.5 * torch.randn((M, V - case["padded"]), generator=g, device="cuda")
        values, index = torch.topk(teacher, k, dim=1)
        if case["padded"]:
            z[:, V - case["padded"]:V] = float("-inf")  # columns that only fill up the matrix
        index = index.to(torch.int32)
        if case["ragged"]:
            length = torch.randint(0, k + 1, (M, 1), generator=g, device="cuda")
            length[M - M // 16:] = 0  # the end of a padded batch
            index[torch.arange(k, device="cuda")[None, :] >= length] = -1
        s["z"] = z.to(DTYPE[case["dtype"]])
        s["values"], s["index"] = values.contiguous(), index.contiguous()
        s["row_scale"] = torch.rand(M, generator=g, device="cuda") / M
        if case["mode"] == "backward":
            z64 = s["z"][:, :V].float()
            largest = z64.amax(1)
            total = torch.logsumexp((z64 - largest[:, None]) / T, 1)
            s["stat"] = torch.stack((largest, total), 1).contiguous()
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------

def _activation(y, act):
    if act == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if act == "hswish":
        return y * (y + 3.0).clamp(0.0, 6.0) / 6.0
    return y


def _plain_quantize(s):
    c, out = s["case"], {}
    if c["rowwise"]:
        out["q"], out["scale"] = _quantized(s["x"], c["format"], c["block"])
    if c["transposed"]:
        out["qt"], out["scale_t"] = _quantized(s["x"].t(), c["format"], c["block"])
    return out


def _plain_linear(s):
    c = s["case"]
    M, K, C = c["M"], c["K"], c["C"]
    x = s["x"].view(F8[c["x_format"]])[:, :C].float() * s["sx"].repeat_interleave(128, 0)[:C].t()
    sw = s["sw"].repeat_interleave(128, 0)[:C].t().repeat_interleave(c["w_block"], 0)[:K]
    w = s["w"].view(F8[c["w_format"]])[:K, :C].float() * sw
    y = torch.matmul(x, w.t())
    if s["bias"] is not None:
        y = y + s["bias"][:K]
    return _activation(y, c["act"]).to(DTYPE[c["y_dtype"]])


def _plain_top(s):
    values, index = torch.sort(s["z"].float(), dim=1, descending=True, stable=True)  # stable: equal values by their index
    k = s["case"]["k"]
    return {"values": values[:, :k].contiguous(), "index": index[:, :k].to(torch.int32)}


def _plain_distill(s):
    c = s["case"]
    V, T = c["V"], c["temperature"]
    z = s["z"][:, :V].float()
    used = (s["index"] >= 0) & (s["index"] < V) & (s["values"] > float("-inf"))
    any_used = used.any(1, keepdim=True)
    at = torch.where(used, s["index"], torch.zeros_like(s["index"])).long()
    t = torch.where(used, s["values"] / T, torch.full_like(s["values"], float("-inf")))
    t = torch.where(any_used, t - t.amax(1, keepdim=True), t)
    p = torch.exp(t)
    p = torch.where(any_used, p / p.sum(1, keepdim=True), torch.zeros_like(p))
    out = {}
    if c["mode"] == "backward":
        largest, total = s["stat"][:, :1], s["stat"][:, 1:]
    else:
        largest = z.amax(1, keepdim=True)
        total = torch.log(torch.exp((z - largest) / T).sum(1, keepdim=True))
        log_q = (torch.gather(z, 1, at) - largest) / T - total
        term = torch.where(p > 0, p * (torch.log(p) - log_q), torch.zeros_like(p))
        out["loss"] = T * T * term.sum(1)
        out["stat"] = torch.cat((largest, total), 1)
    if c["mode"] != "loss":
        d = torch.exp((z - largest) / T - total)
        d.scatter_add_(1, at, -p)
        d *= torch.where(any_used, s["row_scale"][:, None] * T, torch.zeros_like(largest))
        out["dz"] = d.to(DTYPE[c["dtype"]])
    return out


def _own_quantize(s, sgs, stream):
    c, x = s["case"], s["x"]
    R, C, block = c["rows"], c["cols"], c["block"]
    d = sgs.QuantizeF8Desc(rows=R, cols=C, dtype=sgs.SGS_BF16 if c["dtype"] == "bf16" else sgs.SGS_F32,
                           format=sgs.SGS_E4M3 if c["format"] == "e4m3" else sgs.SGS_E5M2, block_rows=block)
    f8, out = F8[c["format"]], {}
    q = scale = qt = scale_t = None
    if c["rowwise"]:
        q = torch.empty((R, _round16(C)), dtype=f8, device="cuda")
        scale = torch.empty((_blocks(C), R if block == 1 else _blocks(R)), dtype=torch.float32, device="cuda")
        out["q"], out["scale"] = q[:, :C], scale
    if c["transposed"]:
        qt = torch.empty((C, _round16(R)), dtype=f8, device="cuda")
        scale_t = torch.empty((_blocks(R), C if block == 1 else _blocks(C)), dtype=torch.float32, device="cuda")
        out["qt"], out["scale_t"] = qt[:, :R], scale_t
    address = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    sgs.quantize_f8(d, x.data_ptr(), address(q), address(scale), address(qt), address(scale_t), stream)
    return out


def _own_linear(s, sgs, stream):
    c = s["case"]
    fmt = {"e4m3": sgs.SGS_E4M3, "e5m2": sgs.SGS_E5M2}
    d = sgs.LinearF8Desc(M=c["M"], K=c["K"], C=c["C"], Kmax=c["Kmax"], Cmax=c["Cmax"], x_format=fmt[c["x_format"]], w_format=fmt[c["w_format"]],
                         w_block_rows=c["w_block"], y_dtype=sgs.SGS_BF16 if c["y_dtype"] == "bf16" else sgs.SGS_F32, act=ACTS[c["act"]])
    y = torch.empty((c["M"], c["K"]), dtype=DTYPE[c["y_dtype"]], device="cuda")
    sgs.linear_f8(d, s["x"].data_ptr(), s["sx"].data_ptr(), s["w"].data_ptr(), s["sw"].data_ptr(),
                  s["bias"].data_ptr() if s["bias"] is not None else 0, y.data_ptr(), stream)
    return y


def _own_top(s, sgs, stream):
    c = s["case"]
    d = sgs.TopLogitsDesc(rows=c["M"], classes=c["V"], top=c["k"], dtype=sgs.SGS_BF16 if c["dtype"] == "bf16" else sgs.SGS_F32)
    values = torch.empty((c["M"], c["k"]), dtype=torch.float32, device="cuda")
    index = torch.empty((c["M"], c["k"]), dtype=torch.int32, device="cuda")
    sgs.top_logits(d, s["z"].data_ptr(), values.data_ptr(), index.data_ptr(), stream)
    return {"values": values, "index": index}


def _own_distill(s, sgs, stream):
    c = s["case"]
    d = sgs.DistillDesc(rows=c["M"], classes=c["V"], top=c["k"], ldz=c["ld"], dtype=sgs.SGS_BF16 if c["dtype"] == "bf16" else sgs.SGS_F32,
                        temperature=c["temperature"], grad_scale=1.0)
    dz = torch.empty((c["M"], c["V"]), dtype=DTYPE[c["dtype"]], device="cuda") if c["mode"] != "loss" else None
    d.lddz = c["V"]
    if c["mode"] == "backward":
        sgs.distill_backward(d, s["z"].data_ptr(), s["values"].data_ptr(), s["index"].data_ptr(), s["stat"].data_ptr(), s["row_scale"].data_ptr(),
                             dz.data_ptr(), stream)
        return {"dz": dz}
    loss = torch.empty(c["M"], dtype=torch.float32, device="cuda")
    stat = torch.empty((c["M"], 2), dtype=torch.float32, device="cuda")
    sgs.distill(d, s["z"].data_ptr(), s["values"].data_ptr(), s["index"].data_ptr(), s["row_scale"].data_ptr(), loss.data_ptr(), stat.data_ptr(),
                dz.data_ptr() if dz is not None else 0, stream)
    out = {"loss": loss, "stat": stat}
    if dz is not None:
        out["dz"] = dz
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2306_17266_b200 as sgs
        call = {"quantize": _own_quantize, "linear": _own_linear, "top": _own_top, "distill": _own_distill}[kind]
        return call(state, sgs, torch.cuda.current_stream().cuda_stream)
    return {"quantize": _plain_quantize, "linear": _plain_linear, "top": _plain_top, "distill": _plain_distill}[kind](state)


def work(case):
    kind = case["kind"]
    size = {"bf16": 2, "f32": 4}
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        sides = int(case["rowwise"]) + int(case["transposed"])
        per = 128 if case["block"] == 1 else 16384
        return {"bytes": n * size[case["dtype"]] + sides * (n + 4 * n / per), "flops": n * (1 + sides)}
    if kind == "linear":
        M, K, C = case["M"], case["K"], case["C"]
        scales = 4 * _blocks(C) * (M + (K if case["w_block"] == 1 else _blocks(K)))
        return {"bytes": M * C + K * C + scales + M * K * size[case["y_dtype"]] + (4 * K if case["bias"] else 0), "flops": 2 * M * K * C}
    n, lists = case["M"] * case["V"] * size[case["dtype"]], 8 * case["M"] * case["k"]
    if kind == "top":
        return {"bytes": n + lists, "flops": case["M"] * case["V"]}
    passes = 1 if case["mode"] == "loss" else 2
    return {"bytes": passes * n + lists + 12 * case["M"], "flops": 4 * passes * case["M"] * case["V"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------

def _exact_codes(x, format, block):
    x = x.double()
    R, C = x.shape
    fine = torch.isfinite(x)
    size = torch.where(fine, x.abs(), torch.zeros_like(x))
    size = torch.nn.functional.pad(size, (0, -C % 128, 0, -R % block))
    largest = size.reshape(size.shape[0] // block, block, size.shape[1] // 128, 128).amax(3).amax(1)
    limit = 1.75 * 2.0 ** TOP_EXPONENT[format]
    e = torch.ceil(torch.log2(largest / limit)).clamp(min=-126)
    e = torch.where(largest > limit * torch.exp2(e), e + 1, e)           # (the logarithm may be off by its own rounding)
    e = torch.where((e > -126) & (largest <= limit * torch.exp2(e - 1)), e - 1, e)
    scale = torch.exp2(e)
    v = x / scale.repeat_interleave(block, 0)[:R].repeat_interleave(128, 1)[:, :C]
    bits, least = (3, -6) if format == "e4m3" else (2, -14)
    exponent = torch.frexp(v)[1].double() - 1
    step = torch.exp2(exponent.clamp(min=least) - bits)
    return torch.where(fine, torch.round(v / step) * step, torch.full_like(v, float("nan"))), scale.t().contiguous()


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        out = {}
        if case["rowwise"]:
            out["q"], out["scale"] = _exact_codes(s["x"], case["format"], case["block"])
        if case["transposed"]:
            out["qt"], out["scale_t"] = _exact_codes(s["x"].t(), case["format"], case["block"])
        return out
    if kind == "linear":
        M, K, C = case["M"], case["K"], case["C"]
        y = torch.zeros((M, K), dtype=torch.float64, device="cuda")
        xq, wq = s["x"].view(F8[case["x_format"]]).double(), s["w"].view(F8[case["w_format"]]).double()
        step = 2048
        for c0 in range(0, C, step):  # (whole blocks of the reduction at a time)
            n = min(step, C - c0)
            b0, nb = c0 // 128, _blocks(n)
            sx = s["sx"][b0:b0 + nb].double()
            sw = s["sw"][b0:b0 + nb].double()[:, torch.arange(K, device="cuda") // case["w_block"]]
            each = torch.arange(n, device="cuda") // 128
            y += (xq[:, c0:c0 + n] * sx[each].t()) @ (wq[:K, c0:c0 + n] * sw[each].t()).t()
        if s["bias"] is not None:
            y += s["bias"][:K].double()
        if case["act"] == "relu":
            y = y.clamp(min=0)
        elif case["act"] == "hswish":
            y = y * (y + 3).clamp(min=0, max=6) / 6
        return y
    if kind == "top":
        return {"values": torch.topk(s["z"].double(), case["k"], dim=1)[0], "index": None}
    V, T = case["V"], case["temperature"]
    out = {}
    z = s["z"][:, :V].double()
    log_q = torch.log_softmax(z / T, 1)
    index = s["index"].long()
    t = (s["values"].double() / T).masked_fill(index < 0, float("-inf"))
    filled = index.amax(1) >= 0
    p = torch.zeros_like(t)
    p[filled] = torch.softmax(t[filled], 1)
    if case["mode"] != "backward":
        cross = p * (torch.log(p.clamp(min=1e-300)) - log_q.gather(1, index.clamp(min=0)))
        out["loss"] = T * T * cross.masked_fill(p == 0, 0).sum(1)
        largest = z.max(1)[0]
        out["stat"] = torch.stack((largest, torch.logsumexp((z - largest[:, None]) / T, 1)), 1)
    if case["mode"] != "loss":
        target = torch.zeros_like(z).scatter_add_(1, index.clamp(min=0), p)
        d = (log_q.exp() - target) * (T * s["row_scale"].double())[:, None]
        d[~filled] = 0
        out["dz"] = d
    return out
