"""A workspace that is too small when a call is captured: the graph has scratch of its own, and the workspace stays one that
eager calls can use before the graph is first replayed and after it is gone."""
import os
import subprocess
import sys

import pytest
import torch

import synth
from test_gpu_serving import _gen, make_batch, objects

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _attention(B):
    b = make_batch([1] * 30, [900] * 30, 64, 1, 256, torch.bfloat16, 3)
    cache, batch = objects(B, b)
    q = torch.randn(30, 4, 256, device="cuda", generator=_gen(1)).bfloat16()
    return lambda ws: B.paged_attention(cache, batch, q, ws=ws)


def _linear(B):
    _, x, _ = synth.activations(40, 1152, 8, seed=3)
    _, w = synth.weight(2304, 1152, seed=3)
    x = x.cuda()
    q = B.prepare_weights(w.cuda(), B.act_absmax(x))
    return lambda ws: B.linear(q, x, ws=ws)


@pytest.mark.parametrize("make", [_attention, _linear])
def test_capture_with_a_fresh_workspace(B, make):
    call = make(B)
    want = call(B.Workspace())
    ws = B.Workspace()
    before = ws.buf.data_ptr()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = call(ws)
    assert ws.buf.data_ptr() == before  # not memory of the graph's
    assert torch.equal(call(ws), want)
    for _ in range(3):
        captured.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, want) and torch.equal(call(ws), want)
    del g, captured
    assert torch.equal(call(ws), want)
    B.workspace_check(ws)


FIRST_CALL = """
import torch
import synth
from paper_2608_28003_gb300 import binding as B
x = synth.activations(40, 1152, 8, seed=3)[1].cuda()
q = B.prepare_weights(synth.weight(2304, 1152, seed=3)[1].cuda(), B.act_absmax(x))
assert not B._DEFAULT_WS
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    y = B.linear(q, x)
assert not B._DEFAULT_WS  # no memory of the graph's for eager calls
want = B.linear(q, x, ws=B.Workspace())
assert torch.equal(B.linear(q, x), want)
for _ in range(3):
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
"""


def test_a_process_whose_first_call_is_captured():
    r = subprocess.run([sys.executable, "-c", FIRST_CALL], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
