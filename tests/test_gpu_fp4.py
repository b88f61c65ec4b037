"""Floating point of 4 bits on the GPU against the 64-bit oracle: quantisation of rows and back, bit for bit, and the linear."""
import numpy as np
import pytest
import torch

from oracle import fp4 as O4

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    from paper_2608_28003_gb300 import build
    build.build()
    from paper_2608_28003_gb300 import binding
    return binding


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _np(t):
    return t.detach().double().cpu().numpy()


def _rows(rows, k, dt, seed, spread=3.0):
    """Rows of very different sizes with a few large columns, some rows of zeros, and ties by construction."""
    x = torch.randn(rows, k, device="cuda", generator=_gen(seed))
    x *= torch.exp(spread * torch.randn(rows, 1, device="cuda", generator=_gen(seed + 1)))
    x[:, ::17] *= 20
    if rows > 2:
        x[1] = 0
        x[2] = torch.randint(-12, 13, (k,), device="cuda", generator=_gen(seed + 2)) * 0.25  # on the borders
        x[2, 0] = 6.0
        x[-1, : k // 2] = 0
    return x.to(DT[dt])


def _check_matrix(q, x, block):
    c, s, r = O4.quantise(_np(x), block)
    got = O4.unpack(q.codes.cpu().numpy())
    np.testing.assert_array_equal(q.block_scales().cpu().numpy(), s)
    if block == 16:
        np.testing.assert_array_equal(_np(q.row_scale), r)
    np.testing.assert_array_equal(O4.values_of(got), O4.values_of(c))
    pad = q.scales.view(-1, 4 * -(-q.k // block // 4) * 128)  # bytes of no row or block
    assert int((pad != 0).sum()) == int((s != 0).sum())
    return O4.dequantise(c, s, r, block)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,k", [(1, 32), (3, 64), (5, 96), (33, 512), (130, 544), (7, 1152), (129, 6912), (2, 16384),
                                    (3, 17440), (2, 65536)])
def test_quantise(B, rows, k, dt, block):
    x = _rows(rows, k, dt, rows + k, 1.0 if dt == "f16" else 3.0)
    q = B.fp4_quantize(x, block)
    want = _check_matrix(q, x, block)
    y = B.fp4_dequantize(q, torch.float32)
    np.testing.assert_array_equal(_np(y), want)
    if dt != "f32":  # six significant bits: exact in bf16, and in fp16 within its range
        np.testing.assert_array_equal(_np(B.fp4_dequantize(q, DT[dt])), want)
    assert torch.equal(B.fp4_dequantize(q, torch.float16), y.half())  # rounded once


@pytest.mark.parametrize("block", [16, 32])
def test_quantise_the_ends_of_the_range(B, block):
    big = torch.finfo(torch.float32).max
    x = torch.zeros(8, 64, device="cuda")
    x[0, 5], x[0, 40] = big, -big / 3
    x[1, 3], x[1, 33] = 2.0 ** -149, -2.0 ** -140
    x[2, 1] = 2.0 ** -126
    x[3, 9], x[3, 60] = 1e38, 1e-38
    x[4] = 2688.0
    x[5, 0] = float(np.nextafter(np.float32(2688), np.float32(3000)))
    x[6, 0], x[6, 16], x[6, 17], x[6, 48] = float("nan"), float("-inf"), 1e30, 3.0
    x[7, 63] = float("inf")
    q = B.fp4_quantize(x, block)
    want = _check_matrix(q, x, block)
    with np.errstate(over="ignore"):
        want32 = want.astype(np.float32)  # the largest number's value lies beyond the type
    np.testing.assert_array_equal(_np(B.fp4_dequantize(q, torch.float32)), want32.astype(np.float64))
    assert np.isnan(want[6, :16]).all() and np.isnan(want[6, 16:32]).all() and not np.isnan(want[6, 48:]).any()


def test_every_bf16_is_decided_right(B):
    """Every finite bf16 number as a block's largest beside its half, and as any smaller one."""
    bits = torch.arange(0, 0x7f80, dtype=torch.int32)
    top = (bits << 16).view(torch.float32).double().numpy()
    x = np.zeros((len(top), 32), np.float32)
    x[:, 0], x[:, 1], x[:, 17] = top, top / 2, top
    x[:, 2:16] = top[:, None] * np.random.default_rng(1).integers(0, 257, (len(top), 14)) / 256
    x = torch.from_numpy(x).cuda().bfloat16()
    for block in (16, 32):
        _check_matrix(B.fp4_quantize(x, block), x, block)


@pytest.mark.parametrize("p", [0, -60, 37, 100])
def test_borders_of_every_scale(B, p):
    """fp32 rows with, for every e4m3 scale, the seven borders of its codes and the numbers next to them on both sides, and blocks whose
    largest magnitude is on and beside every border of the scales."""
    near = lambda x: [np.nextafter(np.float32(x), np.float32(0)), np.float32(x), np.nextafter(np.float32(x), np.float32(1e30))]  # noqa: E731
    blocks = []
    for s in O4.E4M3[1:]:
        borders = [v for b in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0) for v in near(b * s)]
        for part in (borders[:11], borders[11:]):
            blocks.append([6 * s] + part + [0.0] * (15 - len(part)))
    for mid in (O4.E4M3[1:] + O4.E4M3[:-1]) / 2:
        for top in near(6 * mid):
            blocks.append([top, -top] + [top * f for f in np.linspace(0, 1, 14)])
    x = np.array(blocks, np.float32)
    x[1::2] *= -1
    first = np.zeros_like(x)
    first[:, 0] = 2000.0  # keeps the row's scale at 2^p
    x = np.concatenate([first, x], 1) * np.float32(2.0 ** p)
    x = torch.from_numpy(x).cuda()
    q = B.fp4_quantize(x, 16)
    assert (q.row_scale == 2.0 ** p).all()
    _check_matrix(q, x, 16)


def test_quantise_views_and_outputs(B):
    wide = torch.randn(9, 3, 128, device="cuda", generator=_gen(1)).bfloat16()
    x = wide[:, 1, :64]
    for block in (16, 32):
        q = B.fp4_quantize(x, block)
        assert torch.equal(B.fp4_dequantize(q), B.fp4_dequantize(B.fp4_quantize(x.contiguous(), block)))
        out = torch.full((9, 96), 7.0, device="cuda", dtype=torch.bfloat16)
        assert B.fp4_dequantize(q, out=out[:, 8:72]).data_ptr() == out[:, 8:72].data_ptr()
        assert (out[:, :8] == 7).all() and (out[:, 72:] == 7).all() and torch.equal(out[:, 8:72], B.fp4_dequantize(q))
    e = B.fp4_quantize(x[:0])
    assert B.fp4_dequantize(e).shape == (0, 64)
    with pytest.raises(ValueError):
        B.fp4_quantize(x, 8)
    with pytest.raises(ValueError):
        B.fp4_quantize(x.t())
    with pytest.raises(B.W8A8Error):
        B.fp4_quantize(wide[:, 1, :40])  # k is no multiple of 32
    with pytest.raises(B.W8A8Error):
        B.fp4_quantize(wide.view(9, -1)[:, 4:68])  # 8 bytes from a boundary
    with pytest.raises(ValueError):
        B.fp4_dequantize(q, torch.float32, out=out[:, :64])


# -------------------------------------------------------------------------------------- linear
def _bound(want, mass, k, dt):
    """Half a step of the result (of fp16 also half its smallest), three fp32 roundings after the sum, and an fp32 sum of k
    products in any order: k 2^-23 of the sum of their magnitudes, which covers sums that are cut off instead of rounded."""
    eps = torch.finfo(dt).eps / 2
    return (eps + 2.0 ** -21) * np.abs(want) + (k * 2.0 ** -23 + 2.0 ** -22) * mass + (2.0 ** -25 if dt == torch.float16 else 1e-38)


def _check_linear(y, xq, wq, bias, k):
    want, mass = O4.linear(xq, wq, bias)
    if bias is not None:
        mass = mass + np.abs(bias)
    err = np.abs(_np(y) - want) - _bound(want, mass, k, y.dtype)
    assert err.max() <= 0, (float(err.max()), np.argwhere(err > 0)[:4].tolist())


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("m,n,k,dt,out,with_bias", [
    (1, 1, 32, "bf16", "bf16", False), (1, 127, 64, "f16", "f32", True), (2, 129, 96, "bf16", "f16", True),
    (3, 300, 1152, "bf16", "bf16", False), (8, 256, 416, "f32", "bf16", True), (9, 1152, 6912, "bf16", "bf16", False),
    (16, 4099, 1152, "bf16", "f32", False), (17, 640, 288, "f16", "f16", False), (33, 1536, 1152, "bf16", "bf16", True),
    (64, 1152, 1024, "bf16", "bf16", False), (100, 777, 2080, "f32", "f32", True), (128, 128, 256, "bf16", "bf16", False),
    (129, 1152, 6912, "f16", "f16", True), (255, 2304, 544, "bf16", "bf16", False), (300, 1000, 1152, "bf16", "bf16", True),
    (513, 6912, 320, "bf16", "bf16", False), (1030, 7000, 544, "bf16", "bf16", True), (771, 10007, 160, "f16", "f32", False),
    (2048, 4800, 96, "bf16", "f16", True), (1030, 5500, 544, "bf16", "bf16", True), (771, 7001, 160, "f16", "f32", False),
    (1793, 3900, 96, "bf16", "f16", True), (2047, 7000, 288, "bf16", "bf16", False), (49, 1152, 6912, "bf16", "bf16", True),
    (30, 130, 2304, "bf16", "f32", False), (60, 1000, 1024, "f32", "f32", True), (90, 515, 2048, "f16", "f16", True)])
def test_linear(B, m, n, k, dt, out, with_bias, block):
    x = torch.randn(m, k, device="cuda", generator=_gen(m + n)).to(DT[dt])
    x[:, ::29] *= 20
    w = (torch.randn(n, k, device="cuda", generator=_gen(k)) * 0.05).to(DT[dt])
    bias = torch.randn(n, device="cuda", generator=_gen(2)) if with_bias else None
    wq = B.fp4_quantize(w, block)
    y = B.fp4_linear(wq, x, bias=bias, dtype=DT[out])
    assert y.shape == (m, n) and y.dtype == DT[out]
    xv, wv = (_np(B.fp4_dequantize(B.fp4_quantize(t, block), torch.float32)) for t in (x, w))
    _check_linear(y, xv, wv, None if bias is None else _np(bias), k)
    assert torch.equal(B.fp4_linear(wq, x, bias=bias, dtype=DT[out]), y)  # the same bits every time


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_linear_rows_do_not_depend_on_others(B, m, block):
    """A row's result is the formula's whatever the other rows hold; NaN blocks reach their row or channel alone."""
    n, k = 200, 480
    x = torch.randn(m, k, device="cuda", generator=_gen(1)).bfloat16()
    w = torch.randn(n, k, device="cuda", generator=_gen(2)).bfloat16()
    x[-1, 100] = float("inf")
    w[7, 479], w[130, 0] = float("nan"), float("-inf")
    y = B.fp4_linear(B.fp4_quantize(w, block), x)
    xv, wv = (_np(B.fp4_dequantize(B.fp4_quantize(t, block), torch.float32)) for t in (x, w))
    nan = np.isnan(xv).any(1)[:, None] | np.isnan(wv).any(1)[None, :]
    got = _np(y)
    assert np.array_equal(np.isnan(got), nan) and nan[:, 7].all() and nan[-1].all()
    want, mass = O4.linear(np.nan_to_num(xv), np.nan_to_num(wv))
    assert (np.abs(got - want) <= _bound(want, mass, k, torch.bfloat16))[~nan].all()


def test_linear_powers_of_two_are_exact(B):
    """Small whole numbers: every product and sum is exact, and a scale of rows and channels only moves the point."""
    for m, n, k in ((4, 96, 128), (130, 260, 1024)):
        x = torch.randint(-6, 7, (m, k), device="cuda", generator=_gen(1)).float()
        x[x.abs() == 5] = 6
        w = torch.randint(-4, 5, (n, k), device="cuda", generator=_gen(2)).float()
        x[:, ::32], w[:, ::32] = 6, 4
        x[:, 16::32], w[:, 16::32] = 6, 4
        e = torch.randint(-20, 20, (m, 1), device="cuda", generator=_gen(3))
        f = torch.randint(-20, 20, (n, 1), device="cuda", generator=_gen(4))
        want = _np(x) @ _np(w).T * 2.0 ** (_np(e) + _np(f).T)
        for block in (16, 32):
            if block == 16:  # scales that are powers of two: 6 -> 1 (row scale 2^p, scale 2^-p)
                wq = B.fp4_quantize(torch.ldexp(w, f), 16)
                if not torch.equal(B.fp4_dequantize(wq, torch.float32), torch.ldexp(w, f)):
                    wq = B.fp4_tensor(B.fp4_quantize(w, 32).codes, torch.full((n, k // 16), 56, dtype=torch.uint8, device="cuda"),
                                      torch.ldexp(torch.ones(n, device="cuda"), f[:, 0]))
            else:
                wq = B.fp4_quantize(torch.ldexp(w, f), 32)
            xs = torch.ldexp(x, e)
            xv = _np(B.fp4_dequantize(B.fp4_quantize(xs, block), torch.float32))
            wv = _np(B.fp4_dequantize(wq, torch.float32))
            got = _np(B.fp4_linear(wq, xs, dtype=torch.float32))
            np.testing.assert_array_equal(got, xv @ wv.T)
            if block == 32:
                np.testing.assert_array_equal(got, want)


def test_linear_weight_quantised_elsewhere(B):
    """One scale for all rows that is no power of two, and a weight whose scales come as a plain matrix."""
    n, k = 200, 256
    codes = torch.randint(0, 256, (n, k // 2), device="cuda", generator=_gen(1), dtype=torch.int32).to(torch.uint8)
    for block, scales, row in ((16, torch.randint(20, 90, (n, k // 16), device="cuda", generator=_gen(2)), torch.tensor(0.0123)),
                               (32, torch.randint(100, 140, (n, k // 32), device="cuda", generator=_gen(2)), None)):
        w = B.fp4_tensor(codes, scales.to(torch.uint8), None if row is None else row.cuda())
        wv = O4.dequantise(O4.unpack(codes.cpu().numpy()), scales.cpu().numpy().astype(np.uint8),
                           None if row is None else np.full(n, np.float32(0.0123)), block)
        x = torch.randn(6, k, device="cuda", generator=_gen(3)).bfloat16()
        xv = _np(B.fp4_dequantize(B.fp4_quantize(x, block), torch.float32))
        _check_linear(B.fp4_linear(w, x, dtype=torch.float32), xv, wv, None, k)


@pytest.mark.parametrize("m", [4, 150])
def test_linear_scales_at_their_ends(B, m):
    """Powers of two from 2^-127 to 2^127 as scales: blocks of zeros under the largest add nothing, large ones meet small rows."""
    n, k = 130, 160
    codes = torch.randint(0, 256, (n, k // 2), device="cuda", generator=_gen(1), dtype=torch.int32).to(torch.uint8)
    scales = torch.full((n, k // 32), 127, dtype=torch.uint8, device="cuda")
    scales[:, 0], scales[:, 1], scales[:, 2], scales[:, 3] = 254, 254, 0, 1
    codes[:, :16] = 0x80  # 0 and -0
    x = torch.randn(m, k, device="cuda", generator=_gen(2))
    x[:, 32:64] *= 2.0 ** -120   # under 2^127
    x[:, 64:128] *= 2.0 ** 120   # under 2^-127 and 2^-126
    xq = B.fp4_quantize(x.bfloat16(), 32)
    w = B.fp4_tensor(codes, scales)
    xv = _np(B.fp4_dequantize(xq, torch.float32))
    wv = O4.dequantise(O4.unpack(codes.cpu().numpy()), scales.cpu().numpy(), None, 32)
    with np.errstate(over="ignore"):  # 4 and 6 times 2^127 are beyond fp32: rounded, infinite
        np.testing.assert_array_equal(_np(B.fp4_dequantize(w, torch.float32)), wv.astype(np.float32))
    _check_linear(B.fp4_linear(w, x.bfloat16(), dtype=torch.float32), xv, wv, None, k)


def test_linear_views_and_refusals(B):
    w = B.fp4_quantize(torch.randn(72, 64, device="cuda", generator=_gen(1)).bfloat16())
    wide = torch.randn(9, 3, 128, device="cuda", generator=_gen(2)).bfloat16()
    x = wide[:, 2, :64]
    want = B.fp4_linear(w, x.contiguous())
    assert torch.equal(B.fp4_linear(w, x), want) and want.dtype == torch.bfloat16
    for dt in (torch.bfloat16, torch.float16, torch.float32):
        out = torch.full((9, 80), 7.0, device="cuda", dtype=dt)
        view = out[:, :72]
        B.fp4_linear(w, x, out=view)
        assert (out[:, 72:] == 7).all() and torch.equal(view, B.fp4_linear(w, x, dtype=dt))
    odd = B.fp4_quantize(torch.randn(71, 64, device="cuda", generator=_gen(1)).bfloat16())
    out = torch.full((9, 75), 7.0, device="cuda", dtype=torch.bfloat16)  # rows that begin anywhere
    B.fp4_linear(odd, x, out=out[:, :71])
    assert (out[:, 71:] == 7).all() and torch.equal(out[:, :71], B.fp4_linear(odd, x))
    assert B.fp4_linear(w, x[:0]).shape == (0, 72)
    for bad in (lambda: B.fp4_linear(w, wide[:, 0]), lambda: B.fp4_linear(w, x, bias=torch.zeros(71, device="cuda")),
                lambda: B.fp4_linear(w, x.int()), lambda: B.fp4_linear(w, x, dtype=torch.float64),
                lambda: B.fp4_linear(w, x, out=torch.empty(9, 73, device="cuda", dtype=torch.bfloat16)),
                lambda: B.fp4_linear(B.Fp4Tensor(w.codes, w.scales[:-1].contiguous(), w.row_scale, 16), x),
                lambda: B.fp4_linear(B.Fp4Tensor(w.codes, w.scales, None, 16), x)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.W8A8Error):
        B.fp4_linear(w, torch.empty(9, 68, device="cuda", dtype=torch.bfloat16)[:, :64])  # rows 136 bytes apart


def test_linear_streams_and_graphs(B):
    """Calls on two streams at once, each with scratch of its own, and a captured chain replayed on new inputs."""
    w1 = B.fp4_quantize(torch.randn(1024, 512, device="cuda", generator=_gen(1)).bfloat16())
    w2 = B.fp4_quantize(torch.randn(512, 1024, device="cuda", generator=_gen(2)).bfloat16(), 32)
    xs = [torch.randn(m, 512, device="cuda", generator=_gen(m)).bfloat16() for m in (5, 90)]
    chain = lambda x, s=None: B.fp4_linear(w2, B.fp4_linear(w1, x, stream=s), stream=s)  # noqa: E731
    want = [chain(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[], []]
    for _ in range(20):
        for i, (x, s) in enumerate(zip(xs, streams)):
            got[i].append(chain(x, s))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(y, want[i]) for y in got[i])
    graphs = []
    for x in xs:
        static = x.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = chain(static)
        graphs.append((g, static, y))
    for turn in (0, 1):
        for (g, static, y), x in zip(graphs, xs):
            static.copy_(x * (1 + turn))
            g.replay()
        torch.cuda.synchronize()
        for (g, static, y), x in zip(graphs, xs):
            assert torch.equal(y, chain(x * (1 + turn)))
