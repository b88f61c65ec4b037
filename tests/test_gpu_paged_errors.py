"""Waits that gave up in paged attention are seen whichever workspace a call had: the device's error word, without a GPU
fault.  The bit is written from the host, as a kernel's timeout would leave it, so no wait is made to run out."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import synth

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


class _Raw:
    def __init__(self, ptr):
        self.__cuda_array_interface__ = dict(shape=(1,), typestr="<i4", data=(ptr, False), version=2)


def _word(B):
    p = ctypes.c_void_p()
    assert B.lib().w8a8_paged_attention_error_word(ctypes.byref(p)) == 0
    return torch.as_tensor(_Raw(p.value), device="cuda")


@pytest.mark.parametrize("bits", [1, 2, 4, 7])
def test_reported_once_then_cleared(B, bits):
    B.paged_attention_check()
    word = _word(B)
    word.fill_(bits)
    with pytest.raises(B.W8A8Error) as e:
        B.paged_attention_check()
    assert e.value.status == 6 and "gave up" in str(e.value)
    assert int(word) == 0
    B.paged_attention_check()


def test_a_graph_of_ones_own_can_fetch_the_word(B):
    word, seen = _word(B), torch.zeros(1, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        seen.copy_(word)
    word.fill_(2)
    g.replay()
    torch.cuda.synchronize()
    assert int(seen) == 2
    with pytest.raises(B.W8A8Error):
        B.paged_attention_check()


def test_a_decoders_own_workspaces(B):
    f32, bf, norms = synth.decoder_weights(1, 1152, 256, 512, n_q=4, n_kv=1, seed=2)
    w = {k: [t.cuda() for t in v] if isinstance(v, list) else v.cuda() for k, v in bf.items()}
    n = {k: [torch.from_numpy(a).cuda() for a in v] if isinstance(v, list) else torch.from_numpy(v).cuda()
         for k, v in norms.items()}
    dec = B.Decoder(B.DecoderConfig(max_batch=2, max_seq=64, max_tokens=128, layers=1, inter=256, vocab=512, window=64,
                                    global_layers=(0,), n_q=4, n_kv=1), w, n)
    k, v = (torch.zeros(1, 4, 16, 1, 256, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for new in (1, 20):
        dec.step_paged(torch.arange(new, dtype=torch.int32, device="cuda"), k, v,
                       B.PagedBatch(i32([0, new]), i32([new]), i32([[2, 0, 1, 3]]), max_new=new))
        dec.check()
        B.paged_attention_check()


FIRST_CALL = """
import torch
from paper_2608_28003_gb300 import binding as B
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
k = torch.ones(2, 16, 1, 64, dtype=torch.bfloat16, device="cuda")
q = torch.ones(%d, 2, 64, dtype=torch.bfloat16, device="cuda")
cache, batch = B.PagedCache(k, k), B.PagedBatch(i32([0, %d]), i32([30]), i32([[0, 1]]), max_new=%d)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    y = B.paged_attention(cache, batch, q)
for _ in range(3):
    g.replay()
B.paged_attention_check()
assert bool((y == 1).all())
"""


@pytest.mark.parametrize("new", [1, 20])
def test_a_process_whose_first_call_is_captured(B, new):
    r = subprocess.run([sys.executable, "-c", FIRST_CALL % (new, new, new)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
