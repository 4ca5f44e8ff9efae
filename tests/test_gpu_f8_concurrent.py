"""Every form of the 8-bit float layer, the operators on logits and a stream of SubNets at once, on streams and host threads of their own:
the results are those of the calls one by one (blocks of several kernels share an SM's tensor memory then)."""
import threading

import numpy as np
import pytest
import torch

import paper_2306_17266_b200 as sgs
from paper_2306_17266_b200 import workload as wl
from tests.gpu_util import nets, to_device
from tests.test_gpu_f8_layer import operand
from tests.test_gpu_logits import lists

pytestmark = pytest.mark.gpu

LAYERS = [(1, 8192, 4096), (16, 1000, 2048), (30, 4096, 4096), (64, 1000, 4096), (300, 1000, 8192), (512, 4096, 1024), (12544, 408, 512), (2600, 2700, 1111)]


def all_jobs():
    rng, jobs = np.random.default_rng(0), []
    for M, K, C in LAYERS:
        for wb in (1, 128):
            x, sx, _, _ = operand(rng, M, C, "e4m3", 1, 1.0)
            w, sw, _, _ = operand(rng, K, C, "e4m3", wb, 0.05)
            y = torch.zeros((M, K), device="cuda")
            d = sgs.LinearF8Desc(M=M, K=K, C=C, Kmax=K, Cmax=C, w_block_rows=wb, y_dtype=sgs.SGS_F32)
            jobs.append((lambda st, a=(d, x, sx, w, sw, y): sgs.linear_f8(a[0], *(t.data_ptr() for t in a[1:5]), 0, a[5].data_ptr(), st), [y]))
    for M, V in ((512, 65536), (4, 131072), (2000, 1000)):
        g = torch.Generator(device="cuda").manual_seed(V)
        z = 3 * torch.randn((M, V), generator=g, device="cuda")
        v, i = lists(g, z, 30)
        loss, dz = torch.zeros(M, device="cuda"), torch.zeros((M, V), device="cuda")
        tv, ti = torch.zeros((M, 40), device="cuda"), torch.zeros((M, 40), dtype=torch.int32, device="cuda")
        d = sgs.DistillDesc(rows=M, classes=V, top=30, dtype=sgs.SGS_F32, temperature=2.0, grad_scale=1.0)
        t = sgs.TopLogitsDesc(rows=M, classes=V, top=40, dtype=sgs.SGS_F32)
        jobs.append((lambda st, a=(d, z, v, i, loss, dz): sgs.distill(a[0], *(u.data_ptr() for u in a[1:4]), 0, a[4].data_ptr(), 0, a[5].data_ptr(), st), [loss, dz]))
        jobs.append((lambda st, a=(t, z, tv, ti): sgs.top_logits(a[0], *(u.data_ptr() for u in a[1:]), st), [tv, ti]))
    return jobs


def test_all_at_once():
    jobs = all_jobs()
    _, _, gnet = nets(wl.RESNET, True)
    n, res = 32, 96
    cfgs = wl.uniform_stream(wl.RESNET, n, seed=61)
    x = to_device(wl.make_inputs(n, 1, res, seed=9, bf16=True).reshape(n, res, res, 3), True)
    out = torch.zeros((n, 1000), device="cuda")
    opts = sgs.StreamOpts(cache_enabled=1, window_q=4, concurrency=2, wave=8, use_graphs=1)
    main, streams = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    for call, _ in jobs:
        call(main.cuda_stream)
    gnet.stream_run(cfgs, x.data_ptr(), 1, res, out.data_ptr(), opts, main.cuda_stream)
    torch.cuda.synchronize()
    want, ref = [[o.clone() for o in outs] for _, outs in jobs], out.clone()
    for _ in range(3):
        for o in [out] + [o for _, outs in jobs for o in outs]:
            o.zero_()
        torch.cuda.synchronize()
        errors = []

        def work(k):
            try:
                for _ in range(5):
                    for call, _ in jobs[k::4]:
                        call(streams[k].cuda_stream)
            except Exception as e:  # noqa: BLE001
                errors.append(e)
        threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
        for t in threads:
            t.start()
        gnet.stream_run(cfgs, x.data_ptr(), 1, res, out.data_ptr(), opts, main.cuda_stream)
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert not errors, errors
        assert sgs.device_status() == 0 and torch.equal(out, ref)
        for (_, outs), w in zip(jobs, want):
            for a, b in zip(outs, w):
                assert torch.equal(a, b)
