"""CPU checks of floating point of 4 bits: the oracle against brute force and closed forms, the order of the scales, and every
refusal of the entry points (nothing reaches a GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fp4 as O4


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


# ------------------------------------------------------------------------------------- the oracle
def test_e4m3_table_is_torchs():
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(O4.E4M3, t)
    x = np.concatenate([np.random.default_rng(1).uniform(0, 448, 5000), O4.E4M3, (O4.E4M3[1:] + O4.E4M3[:-1]) / 2,
                        10.0 ** np.linspace(-5, 2, 500)])
    want = torch.tensor(x).float().to(torch.float8_e4m3fn).double().numpy()
    fine = torch.tensor(x).float().double().numpy() == x  # what fp32 holds
    np.testing.assert_array_equal(O4.E4M3[O4.nearest(x, O4.E4M3)][fine], want[fine])


def test_codes_at_the_borders():
    x = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 1e30])
    even = np.array([0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0])
    for s in (1.0, 0.40625, 2.0 ** -20):
        np.testing.assert_array_equal(O4.values_of(O4.codes_of(x * s, s)), even)
        np.testing.assert_array_equal(O4.values_of(O4.codes_of(-x * s, s)), -even)
        up = np.nextafter(x[:7] * s, np.inf)
        np.testing.assert_array_equal(O4.values_of(O4.codes_of(up, s)), [0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
        down = np.nextafter(x[:7] * s, 0)
        np.testing.assert_array_equal(O4.values_of(O4.codes_of(down, s)), [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0])
    assert O4.codes_of(1.0, 0.0) == 0


def test_blocks_by_hand():
    x = np.zeros((2, 64))
    x[0, :4], x[0, 40] = [7.5, -1.0, 3.0, 0.3], 1000.0
    c, s, _ = O4.quantise(x, 32)
    assert list(s[0]) == [127, 127 + 7] and s[1].max() == 0   # 2^(2 - 2), 2^(9 - 2)
    np.testing.assert_array_equal(O4.dequantise(c, s, None, 32)[0, [0, 1, 2, 3, 40]], [6.0, -1.0, 3.0, 0.5, 768.0])
    c, s, r = O4.quantise(x, 16)
    assert list(r) == [0.5, 1.0]  # 1000 <= 2688 / 2, > 2688 / 4
    np.testing.assert_array_equal(O4.E4M3[s[0]], [2.5, 0.0, 320.0, 0.0])  # 7.5 / 6 / 0.5; 1000 / 6 / 0.5 = 333.3
    v = O4.dequantise(c, s, r, 16)[0, [0, 1, 2, 3, 40]]
    np.testing.assert_array_equal(v, [7.5, -1.25, 2.5, 0.0, 960.0])  # 0.3 / 1.25 = 0.24; 3 / 1.25 = 2.4; 6 * 160
    x[0, 0] = np.nan
    c, s, r = O4.quantise(x, 16)
    v = O4.dequantise(c, s, r, 16)
    assert s[0, 0] == 127 and np.isnan(v[0, :16]).all() and np.isfinite(v[0, 16:]).all()


def test_no_value_is_further_than_half_a_step():
    x = np.random.default_rng(2).standard_normal((40, 96)) * 10.0 ** np.random.default_rng(3).uniform(-6, 6, (40, 1))
    for block, most in ((32, 1.0 / 4), (16, 1.0 / 6 + 1.0 / 16)):  # 7.99 -> 6 of 8; a step of 2 at 6 and the scale's half step
        v = O4.dequantise(*O4.quantise(x, block), block)
        top = np.abs(x.reshape(40, -1, block)).max(-1)
        assert (np.abs(v - x).reshape(40, -1, block).max(-1) <= most * top).all()
        w = O4.dequantise(*O4.quantise(v, 32), 32) if block == 32 else v
        np.testing.assert_array_equal(w, v)  # values of powers of two stay what they are
    np.testing.assert_array_equal(O4.unpack(O4.pack(O4.codes_of(x, 0.3))), O4.codes_of(x, 0.3))


# ------------------------------------------------------------------------------------- scales in order
@pytest.mark.parametrize("rows,k,block", [(1, 32, 32), (1, 32, 16), (130, 224, 16), (257, 1152, 32), (128, 64, 16)])
def test_scale_order(B, rows, k, block):
    size = ctypes.c_size_t()
    assert B.lib().w8a8_fp4_scale_bytes(rows, k, block, ctypes.byref(size)) == 0
    g = -(-(k // block) // 4)
    assert size.value == -(-rows // 128) * g * 512
    plain = torch.randint(1, 127, (rows, k // block), dtype=torch.uint8)
    t = B.fp4_tensor(torch.zeros(rows, k // 2, dtype=torch.uint8), plain)
    assert t.block == block and t.scales.numel() == size.value and (t.row_scale is None) == (block == 32)
    assert torch.equal(t.block_scales(), plain) and (t.rows, t.k) == (rows, k)
    for r, j in ((0, 0), (rows - 1, k // block - 1), (rows // 2, k // block // 2)):
        at = ((r // 128) * g + j // 4) * 512 + (r % 32) * 16 + (r // 32) % 4 * 4 + j % 4
        assert t.scales[at] == plain[r, j]
    assert int((t.scales != 0).sum()) == plain.numel()  # the others are 0


# ------------------------------------------------------------------------------------- refusals
P = ctypes.c_void_p(0x10000)


def _q(B, rows=4, k=64, block=16, codes=0x1000, scales=0x2000, row_scale=0x3000):
    return B.Fp4C(rows, k, block, codes, scales, row_scale if block == 16 else None)


@pytest.mark.parametrize("kw,want", [
    (dict(block=8), 1), (dict(k=48), 2), (dict(k=0), 2), (dict(k=65568), 2), (dict(rows=-1), 2), (dict(rows=2 ** 31 - 1), 2), (dict(codes=None), 1),
    (dict(scales=None), 1), (dict(row_scale=None), 1), (dict(codes=0x1008), 3), (dict(scales=0x2004), 3),
    (dict(row_scale=0x3004), 3)])
def test_matrix_refusals(B, kw, want):
    L, q = B.lib(), _q(B, **kw)
    assert L.w8a8_fp4_quantize(0, P, 64, ctypes.byref(q), None) == want
    assert L.w8a8_fp4_dequantize(ctypes.byref(q), 0, P, 65600, None) == want
    assert L.w8a8_fp4_linear(ctypes.byref(q), 0, P, 65600, 3, None, 0, P, 64, P, 1 << 30, None) == want
    assert L.w8a8_last_error()


def test_signed_scales_are_refused(B):
    codes, plain = torch.zeros(3, 32, dtype=torch.uint8), torch.full((3, 4), 130, dtype=torch.uint8)
    with pytest.raises(ValueError, match="no sign"):
        B.fp4_tensor(codes, plain)
    assert B.fp4_tensor(codes, plain[:, :2]).block == 32  # there all of the byte is the exponent


def test_call_refusals(B):
    L, q = B.lib(), _q(B)
    r = ctypes.byref(q)
    assert L.w8a8_fp4_quantize(3, P, 64, r, None) == 1           # type
    assert L.w8a8_fp4_quantize(0, P, 60, r, None) == 2           # row stride
    assert L.w8a8_fp4_quantize(2, P, 62, r, None) == 2
    assert L.w8a8_fp4_quantize(0, None, 64, r, None) == 1
    assert L.w8a8_fp4_quantize(0, ctypes.c_void_p(0x10008), 64, r, None) == 3
    assert L.w8a8_fp4_quantize(0, P, 64, None, None) == 1
    assert L.w8a8_fp4_dequantize(r, 0, P, 56, None) == 2         # rows that overlap
    assert L.w8a8_fp4_dequantize(r, -1, P, 64, None) == 1
    assert L.w8a8_fp4_dequantize(r, 0, None, 64, None) == 1
    out = ctypes.c_void_p(0x20000)
    lin = lambda *a: L.w8a8_fp4_linear(*a)  # noqa: E731
    assert lin(r, 0, P, 64, -1, None, 0, out, 64, P, 1 << 30, None) == 1
    assert lin(r, 4, P, 64, 3, None, 0, out, 64, P, 1 << 30, None) == 1
    assert lin(r, 0, P, 64, 3, None, 3, out, 64, P, 1 << 30, None) == 1
    assert lin(r, 0, P, 63, 3, None, 0, out, 64, P, 1 << 30, None) == 2
    assert lin(r, 0, P, 64, 3, None, 0, out, 3, P, 1 << 30, None) == 2       # Y's rows overlap (N = 4)
    assert lin(r, 0, None, 64, 3, None, 0, out, 64, P, 1 << 30, None) == 1
    assert lin(r, 0, P, 64, 3, None, 0, P, 64, P, 1 << 30, None) == 1        # in place
    assert lin(r, 0, P, 64, 3, ctypes.c_void_p(0x30004), 0, out, 64, P, 1 << 30, None) == 3
    assert lin(r, 0, P, 64, 0, None, 0, None, 64, None, 0, None) == 0        # of nothing
    n = ctypes.c_size_t()
    assert L.w8a8_fp4_linear_workspace_size(3, 4, 64, 16, ctypes.byref(n)) == 0 and n.value > 65536
    assert L.w8a8_fp4_linear_workspace_size(3, 4, 64, 24, ctypes.byref(n)) == 1
    assert L.w8a8_fp4_linear_workspace_size(3, 4, 60, 16, ctypes.byref(n)) == 2
    assert L.w8a8_fp4_linear_workspace_size(-3, 4, 64, 16, ctypes.byref(n)) == 2
    assert L.w8a8_fp4_scale_bytes(4, 64, 16, None) == 1 and L.w8a8_fp4_scale_bytes(4, 40, 16, ctypes.byref(n)) == 2


def _cache(B, **kw):
    f = dict(n_pages=8, page_size=16, n_kv=2, head_dim=128, k_exp=0, v_exp=0, page_stride=2048, slot_stride=128, head_stride=64,
             s_page_stride=256, s_slot_stride=16, s_head_stride=8, k=0x1000, v=0x2000, k_scales=0x3000, v_scales=0x4000)
    f.update(kw)
    return B.PagedCacheFp4C(*f.values())


CACHE_BAD = [(dict(n_pages=0), 1), (dict(page_size=24), 2), (dict(head_dim=96), 2), (dict(n_kv=0), 1), (dict(k_exp=101), 1),
             (dict(v_exp=-101), 1), (dict(page_stride=2056), 2), (dict(slot_stride=48), 2), (dict(head_stride=72), 2),
             (dict(s_page_stride=252), 2), (dict(s_slot_stride=4), 2), (dict(s_head_stride=-8), 2), (dict(k=None), 1),
             (dict(v_scales=None), 1), (dict(k=0x1008), 3), (dict(k_scales=0x3008), 3)]


@pytest.mark.parametrize("kw,want", CACHE_BAD)
def test_cache_refusals(B, kw, want):
    L, c = B.lib(), _cache(B, **kw)
    b = B.PagedBatchC(2, 3, 2, 4, 0x5000, 0x6000, 0x7000)
    t = B.RopeTableC(64, 0, 1.0, 0x8000)
    cp, bp = ctypes.byref(c), ctypes.byref(b)
    assert L.w8a8_fp4_rope_append(ctypes.byref(t), cp, bp, 0, P, 512, 4, P, 512, P, 512, None, None, 1e-6, P, 512, None) == want
    assert L.w8a8_fp4_paged_attention(cp, bp, 0, P, 512, 128, 4, 0.1, 0, ctypes.c_void_p(0x20000), 512, 128, P, 1 << 30,
                                      None) == want
    assert L.w8a8_fp4_paged_values(cp, None, c.n_pages, 0, P, P, None) == want


def test_cached_call_refusals(B):
    L, c = B.lib(), _cache(B)
    b = B.PagedBatchC(2, 3, 2, 4, 0x5000, 0x6000, 0x7000)
    t = B.RopeTableC(64, 0, 1.0, 0x8000)
    cp, bp, tp, o = ctypes.byref(c), ctypes.byref(b), ctypes.byref(t), ctypes.c_void_p(0x20000)
    app = lambda dtype=0, q=P, n_q=4, out=P, stride=512, eps=1e-6, norm=None, table=tp: L.w8a8_fp4_rope_append(  # noqa: E731
        table, cp, bp, dtype, q, 512, n_q, P, 512, P, 512, norm, None, eps, out, stride, None)
    assert app(dtype=2) == 1 and app(q=None) == 1 and app(n_q=0) == 2 and app(out=o, stride=504) == 2 and app(stride=520) == 2
    assert app(eps=float("nan"), norm=P) == 1 and app(table=None) == 1 and app(norm=ctypes.c_void_p(0x30004)) == 3
    wide = B.RopeTableC(144, 0, 1.0, 0x8000)
    assert app(table=ctypes.byref(wide)) == 2
    att = lambda dtype=0, q=P, n_q=4, scale=0.1, window=0, out=o, o_row=512, ws=P, size=1 << 30: \
        L.w8a8_fp4_paged_attention(cp, bp, dtype, q, 512, 128, n_q, scale, window, out, o_row, 128, ws, size, None)  # noqa: E731
    assert att(dtype=2) == 1 and att(n_q=3) == 2 and att(scale=0.0) == 1 and att(scale=float("inf")) == 1 and att(window=-1) == 1
    assert att(out=P) == 1 and att(o_row=256) == 2 and att(q=None) == 1
    n = ctypes.c_size_t()
    assert L.w8a8_fp4_paged_attention_workspace_size(cp, 4, ctypes.byref(n)) == 0 and n.value > 65536
    assert L.w8a8_fp4_paged_attention_workspace_size(cp, 3, ctypes.byref(n)) == 2
    val = lambda pages=None, n=8, dtype=0, k=P, v=P: L.w8a8_fp4_paged_values(cp, pages, n, dtype, k, v, None)  # noqa: E731
    assert val(n=7) == 1 and val(n=-1, pages=P) == 1 and val(dtype=3) == 1 and val(k=ctypes.c_void_p(0x10008)) == 3
    assert val(pages=P, n=0) == 0 and val(k=None, v=None) == 0
    none = B.PagedBatchC(2, 0, 2, 4, None, None, None)  # calls of nothing
    assert L.w8a8_fp4_paged_attention(cp, ctypes.byref(none), 0, None, 512, 128, 4, 0.1, 0, None, 512, 128, None, 0, None) == 0


def test_binding_refusals(B):
    codes = torch.zeros(3, 32, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.fp4_tensor(codes, torch.zeros(3, 3, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.fp4_tensor(codes, torch.zeros(2, 4, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.fp4_tensor(codes.int(), torch.zeros(3, 4, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.fp4_tensor(codes, torch.zeros(3, 2, dtype=torch.uint8), torch.ones(3))
    for call in (lambda: B.fp4_quantize(torch.zeros(3, 64)), lambda: B.fp4_dequantize(B.fp4_tensor(codes, codes[:, :4])),
                 lambda: B.fp4_linear(B.fp4_tensor(codes, codes[:, :4]), torch.zeros(3, 64))):
        with pytest.raises(AssertionError):  # CPU tensors
            call()
    with pytest.raises(ValueError):
        B.fp4_dequantize(B.fp4_tensor(codes, codes[:, :4]), torch.int32)
