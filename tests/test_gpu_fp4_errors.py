"""Waits that gave up in the 4-bit linear are seen whichever workspace a call had, the stream's own and a captured call's included:
the device's error word, without a GPU fault.  The bit is written from the host, as a kernel's timeout would leave it."""
import ctypes
import subprocess
import sys

import pytest
import torch

from test_gpu_paged_errors import ROOT, _Raw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _word(B):
    p = ctypes.c_void_p()
    assert B.lib().w8a8_fp4_linear_error_word(ctypes.byref(p)) == 0
    return torch.as_tensor(_Raw(p.value), device="cuda")


@pytest.mark.parametrize("bits", [1, 2, 4, 7])
def test_reported_once_then_cleared(B, bits):
    B.fp4_linear_check()
    word = _word(B)
    word.fill_(bits)
    B.paged_attention_check()  # another word
    with pytest.raises(B.W8A8Error) as e:
        B.fp4_linear_check()
    assert e.value.status == 6 and "gave up" in str(e.value)
    assert int(word) == 0
    B.fp4_linear_check()


@pytest.mark.parametrize("m", [1, 40, 200])
def test_calls_that_are_well_leave_the_word_alone(B, m):
    g = torch.Generator("cuda").manual_seed(m)
    w = B.fp4_quantize(torch.randn(512, 2304, device="cuda", generator=g).bfloat16())
    x = torch.randn(m, 2304, device="cuda", generator=g).bfloat16()
    want = B.fp4_linear(w, x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = B.fp4_linear(w, x)
    for _ in range(3):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)
    B.fp4_linear_check()
    _word(B).fill_(2)  # of an earlier call: a call after it does not clear it
    assert torch.equal(B.fp4_linear(w, x), want)
    with pytest.raises(B.W8A8Error):
        B.fp4_linear_check()


FIRST_CALL = """
import torch
from paper_2608_28003_gb300 import binding as B
w = B.fp4_quantize(torch.ones(128, 1024, dtype=torch.bfloat16, device="cuda"))
x = torch.ones(%d, 1024, dtype=torch.bfloat16, device="cuda")
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    y = B.fp4_linear(w, x)
for _ in range(3):
    g.replay()
B.fp4_linear_check()
assert bool((y == 1088).all())
"""  # 1 is 6 e4m3(1 / 6) = 6 * 11 / 64 = 1.03125; 1024 times its square is 1089, which bf16's eight bits round to 1088


@pytest.mark.parametrize("m", [1, 100])
def test_a_process_whose_first_call_is_captured(m):
    r = subprocess.run([sys.executable, "-c", FIRST_CALL % m], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
