"""CPU checks of the error queries of paged attention and of a model (nothing reaches a GPU)."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def test_null_arguments(B):
    assert B.lib().w8a8_model_check(None, None) == 1
    assert B.lib().w8a8_paged_attention_error_word(None) == 1


def test_attention_in_place_is_refused(B):
    import ctypes
    P = 0x10000  # an aligned address nothing reads
    c = B.PagedCacheC(0, 4, 16, 2, 128, 4096, 256, 128, P, P)
    b = B.PagedBatchC(2, 3, 2, 4, P, P, P)

    def attn(o, ws):
        return B.lib().w8a8_paged_attention(ctypes.byref(c), ctypes.byref(b), P, 1024, 128, 8, 0.1, 0, o, 1024, 128, ws, 0, None)
    assert attn(P, P) == 1 and b"must not be q" in B.lib().w8a8_last_error()
    assert attn(2 * P, P) != 1


def test_rope_of_more_heads_than_steps_of_32_bits_reach(B):
    import ctypes
    P = 0x10000
    t = B.RopeTableC(16, 0, 1.0, P)

    def rope(heads):
        return B.lib().w8a8_rope(ctypes.byref(t), 0, P, 16, 16, 1, heads, 16, P, 2 * P, 16, 16, None)
    assert rope((1 << 31) - 1) == 2 and rope((1 << 30) + 1) == 2 and b"2^30 heads" in B.lib().w8a8_last_error()
