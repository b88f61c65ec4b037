"""Calls of several host threads on one stream, without workspaces of their own: each call's launches stay together."""
import sys
import threading

import pytest
import torch

import synth
from test_gpu_serving import make_batch, objects

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _fp4(B, m, n, k):
    g = torch.Generator("cuda").manual_seed(m)
    w = B.fp4_quantize(torch.randn(n, k, device="cuda", generator=g).bfloat16(), 16 if m % 2 else 32)
    x = torch.randn(m, k, device="cuda", generator=g).bfloat16()
    out = torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    return lambda: B.fp4_linear(w, x, out=out)


def _w8a8(B, m, n, k):
    x = synth.activations(m, k, 8, seed=m)[1].cuda()
    q = B.prepare_weights(synth.weight(n, k, seed=m)[1].cuda(), B.act_absmax(x))
    out = torch.empty(m, n, device="cuda", dtype=torch.bfloat16)
    return lambda: B.linear(q, x, out=out)


def _attention(B, m, *_):
    b = make_batch([m] * 3, [2000] * 3, 64, 2, 128, torch.bfloat16, m)
    cache, batch = objects(B, b)
    q = torch.randn(b["n_rows"], 8, 128, device="cuda", generator=torch.Generator("cuda").manual_seed(m)).bfloat16()
    out = torch.empty_like(q)
    return lambda: B.paged_attention(cache, batch, q, out=out)


@pytest.mark.parametrize("makes", [[_fp4, _fp4, _fp4], [_fp4, _attention, _fp4], [_w8a8, _w8a8, _w8a8]],
                         ids=["fp4", "fp4 and attention", "w8a8"])
def test_threads_on_one_stream(B, makes):
    calls = [make(B, *s) for make, s in zip(makes, ((17, 512, 1152), (200, 256, 512), (33, 1024, 2304)))]
    want = [c().clone() for c in calls]
    torch.cuda.synchronize()
    bad = [torch.zeros((), dtype=torch.bool, device="cuda") for _ in calls]
    errors, go = [], threading.Barrier(len(calls))

    def work(i):
        try:
            go.wait()
            for n in range(1500):
                y = calls[i]()
                if n % 8 == 0:
                    bad[i] |= (y.view(torch.int16) != want[i].view(torch.int16)).any()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    was = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(was)
    torch.cuda.synchronize()
    assert not errors, errors
    assert not any(bool(b) for b in bad), [bool(b) for b in bad]
