"""defl_mx4_quantize, defl_mx4_dequantize and defl_mx4_gemm on the GPU against the fp64 oracle.

Quantisation is defined to the bit and compared so. Products: every product of two codes is exact in fp32 and so is its scaling by
powers of two; a sum of K terms in fp32, in any order and even if every addition cuts its result off instead of rounding it (2^-23 of
at most the sum of magnitudes S), is within K 2^-23 S; e4m3 scales add two roundings a block (2^-23 S together), the matrices'
scales and alpha three (E = 2^-24 each), bf16 half a unit (2^-8). Where all sums are exact in fp32 the result is compared to the bit.
"""
import numpy as np
import pytest
import torch

from oracle import mx4

BF16, F32 = torch.bfloat16, torch.float32
FORMATS = ["mxfp4", "nvfp4"]


@pytest.fixture(scope="module")
def ctx():
    from paper_2609_21102_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


def _rand(shape, seed, dtype, spread=1.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape[:-1] + (1,)))
    return torch.tensor(x, dtype=torch.float64).to(dtype)


def _same(q, X, fmt):
    """q holds X [b, rows, cols] (blocks along cols) to the bit, padding included."""
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    for i in range(X.shape[0]):
        index, byte, whole = mx4.quantize(X[i], fmt)
        have = np.stack([codes[i] & 15, codes[i] >> 4], axis=2).reshape(index.shape).astype(np.int64)
        bad = mx4.decode_scale(byte, fmt, whole)
        fine = np.repeat(np.isfinite(bad), mx4.BLOCK[fmt], axis=1)          # the codes beside a NaN scale mean nothing
        got = np.where(have >= 8, -(have & 7), have & 7)
        assert np.array_equal(got[fine], index[fine])
        assert np.all(have[:, X.shape[2]:] == 0)
        assert np.array_equal(scales[i], mx4.tiles(byte))
        if fmt == "nvfp4":
            assert float(q.scale[i]) == whole


SHAPES = [(1, 1, 1), (1, 1, 31), (2, 33, 32), (1, 32, 33), (3, 17, 16), (1, 127, 129), (2, 130, 70), (1, 256, 384), (1, 300, 1003), (1, 1003, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantise_to_the_bit(ctx, fmt, dtype, shape):
    X = _rand(shape, 1, dtype).cuda()
    X64 = X.double().cpu().numpy()
    q, qt = ctx.defl_mx4_quantize(X, fmt, both=True)
    _same(q, X64, fmt)
    _same(qt, X64.transpose(0, 2, 1), fmt)
    for a, b in ((q, ctx.defl_mx4_quantize(X, fmt)), (qt, ctx.defl_mx4_quantize(X, fmt, transposed=True))):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    back, backt = ctx.defl_mx4_dequantize(q, F32).double().cpu().numpy(), ctx.defl_mx4_dequantize(qt, BF16).double().cpu().numpy()
    for i in range(shape[0]):
        assert np.array_equal(back[i], mx4.round_trip(X64[i], fmt)) and np.array_equal(backt[i], mx4.round_trip(X64[i].T, fmt))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantise_strides(ctx, fmt, dtype):
    """Rows further apart than they are long, an odd address, batches apart, and a matrix that lies column by column."""
    big = _rand((3, 140, 264), 2, dtype).cuda()
    for X in (big[:, :130, :100], big[:, 3:, 1:200], big[::2, :, 8:136], big[1:2], big.transpose(1, 2), big[:, :100, :77].transpose(1, 2)):
        X64 = X.double().cpu().numpy()
        q, qt = ctx.defl_mx4_quantize(X, fmt, both=True)
        _same(q, X64, fmt)
        _same(qt, X64.transpose(0, 2, 1), fmt)
        _same(ctx.defl_mx4_quantize(X, fmt, transposed=True), X64.transpose(0, 2, 1), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantise_where_it_can_go_wrong(ctx, fmt, dtype):
    """Ties between codes and between scales, zeros of both signs, NaN and Inf, the ends of the range."""
    rng = np.random.default_rng(3)
    n = 256
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, -0.0, -0.25, -5.0, 6.0])
    X = rng.choice(ties, (1, 8 * 32, n))
    X[0, 0:32] *= 1.0625                                     # e4m3 scales with a mantissa
    X[0, 32:64] *= 2.0 ** -20
    X[0, 64:96] = 6.0 * (1 + rng.integers(0, 16, (32, n)) / 16)     # largest magnitudes halfway between e4m3 scales
    X[0, 96] = 0.0
    X[0, 97, ::7] = np.nan
    X[0, 98, 40], X[0, 99, 41] = np.inf, -np.inf
    X[0, 128:160] *= 2.0 ** -126 if fmt == "mxfp4" else 2.0 ** -30
    t = torch.tensor(X).to(dtype).cuda()
    for part in (t, t[:, 64:97], t[:, 128:160], t[:, 96:97], t * 2.0 ** -120, t * 2.0 ** 123, torch.zeros_like(t), torch.full_like(t, float("nan"))):
        part = part.contiguous()
        P = part.double().cpu().numpy()
        q, qt = ctx.defl_mx4_quantize(part, fmt, both=True)
        _same(q, P, fmt)
        _same(qt, P.transpose(0, 2, 1), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", [0, 16, 4])
@pytest.mark.parametrize("shape", [(2, 33, 40), (1, 5, 1000), (1, 3, 4112), (2, 9, 1003)])
def test_dequantise_into_any_place(ctx, fmt, dtype, offset, shape):
    """Results that start on 32, 16 or 4 bytes, rows that do and do not: the values of the codes, and nothing beside them."""
    import ctypes
    from paper_2609_21102_b200 import binding
    q = ctx.defl_mx4_quantize(_rand(shape, 15, F32).cuda(), fmt)
    n, es = int(np.prod(shape)), 2 if dtype == BF16 else 4
    buf = torch.full((n * es + 96,), 0x5a, dtype=torch.uint8, device="cuda")
    ref = (ctypes.c_void_p * 3)(q.codes.data_ptr(), q.scales.data_ptr(), q.scale.data_ptr() if q.scale is not None else None)
    torch.cuda.synchronize()
    rc = binding.lib().defl_mx4_dequantize(ctypes.c_void_p(ctx._handle), ref, *shape, binding.MX4_FORMATS[fmt], ctypes.c_void_p(buf.data_ptr() + 32 + offset),
                                           binding.BF16 if dtype == BF16 else binding.F32)
    torch.cuda.synchronize()
    assert rc == 0
    host = buf.cpu().numpy()
    assert np.all(host[:32 + offset] == 0x5a) and np.all(host[32 + offset + n * es:] == 0x5a)
    got = torch.from_numpy(host[32 + offset:32 + offset + n * es].copy()).view(dtype).double().reshape(shape).numpy()
    codes = q.codes.cpu().numpy()
    for i in range(shape[0]):
        index = np.stack([codes[i] & 15, codes[i] >> 4], axis=2).reshape(shape[1], -1).astype(np.int64)
        value = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])[index & 7] * np.where(index >= 8, -1.0, 1.0)
        scale = mx4.decode_scale(q.plain_scales()[i].cpu().numpy().astype(np.int64), fmt, float(q.scale[i]) if q.scale is not None else 1.0)
        assert np.array_equal(got[i], (value * np.repeat(scale, mx4.BLOCK[fmt], axis=1))[:, :shape[2]])


def _mx(ctx, shape, seed, fmt, dtype=F32, spread=1.0):
    return ctx.defl_mx4_quantize(_rand(shape, seed, dtype, spread).cuda(), fmt)


def _check(ctx, D, A, B, alpha=1.0, scale=1.0):
    a, b = ctx.defl_mx4_dequantize(A, F32).double(), ctx.defl_mx4_dequantize(B, F32).double()
    want = alpha * scale * (a @ b.transpose(1, 2))
    S = abs(alpha * scale) * (a.abs() @ b.abs().transpose(1, 2))
    bound = 1.1 * (A.cols * 2.0 ** -23 + 2.0 ** -22) * S + 1e-44
    if D.dtype == BF16:
        bound = bound * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8
    assert torch.all((D.double() - want).abs() <= bound), float(((D.double() - want).abs() / bound.clamp(min=1e-300)).max())


ROWS = [(1, 1, 64, 32), (1, 1, 6400, 1600), (2, 3, 100, 1003), (1, 8, 700, 5000), (1, 5, 33, 9000), (1, 2, 1, 48), (3, 7, 1600, 96)]
TILES = [(1, 9, 64, 32), (1, 128, 64, 64), (1, 128, 256, 512), (1, 100, 200, 1000), (2, 77, 6400, 1600), (1, 129, 1, 32), (1, 256, 64, 256),
         (1, 256, 256, 1024), (3, 333, 517, 1003), (1, 1024, 768, 768), (2, 2000, 1600, 640), (1, 4100, 6400, 32), (1, 4096, 4097, 300),
         (1, 700, 192, 2048), (5, 260, 330, 80), (1, 16, 20000, 128), (1, 8192, 48, 64),
         (1, 128, 1600, 6400), (2, 40, 130, 5000), (1, 300, 100, 9001), (1, 9, 7, 2300)]          # the last four in parts along K


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("shape", ROWS + TILES)
def test_product_matches_fp64(ctx, fmt, out, shape):
    b, M, N, K = shape
    A, B = _mx(ctx, (b, M, K), 4, fmt), _mx(ctx, (b, N, K), 5, fmt)
    _check(ctx, ctx.defl_mx4_gemm(A, B, out_dtype=out, alpha=0.75), A, B, 0.75)
    assert ctx.defl_device_wait_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shape", ROWS + TILES)
def test_exact_sums(ctx, fmt, shape):
    """Grid values with a six in every block: scales of one, sums of multiples of 1/4 below 36 K < 2^22, exact in fp32 in any order."""
    b, M, N, K = shape
    rng = np.random.default_rng(6)
    vals = np.concatenate([mx4.GRID, -mx4.GRID])

    def make(rows):
        x = rng.choice(vals, (b, rows, K))
        x[:, :, ::16] = 6.0
        return ctx.defl_mx4_quantize(torch.tensor(x, dtype=F32).cuda(), fmt), torch.tensor(x).cuda()
    (A, a), (B, c) = make(M), make(N)
    D = ctx.defl_mx4_gemm(A, B, out_dtype=F32)
    assert torch.equal(D.double(), a @ c.transpose(1, 2))


@pytest.mark.gpu
def test_which_products_go_in_parts(ctx):
    from paper_2609_21102_b200 import binding
    room = lambda *s: binding.lib().defl_mx4_gemm_work_bytes(ctx._h, *s, 0)  # noqa: E731
    for b, M, N, K in TILES[-4:]:
        parts = room(b, M, N, K) / (b * M * ((N + 3) // 4 * 4) * 4)
        assert parts in (2, 3, 4, 5, 6, 7, 8)
    for b, M, N, K in TILES[:-4] + ROWS:
        assert room(b, M, N, K) == 0 or K >= 2048


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("M", [4, 100, 300])
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_result_in_a_larger_buffer(ctx, fmt, out, M, pad):
    """Rows of another stride, at an odd address: what lies between and behind them stays; B shared by the batch."""
    b, N, K = 2, 150 - pad, 224
    A, B = _mx(ctx, (b, M, K), 7, fmt), _mx(ctx, (1, N, K), 8, fmt)
    buf = torch.full((b, M + 5, N + 2 * pad + 2), 123.0, dtype=out, device="cuda")
    D = ctx.defl_mx4_gemm(A, B, out=buf[:, 2:2 + M, pad:pad + N])
    _check(ctx, D, A, B)
    buf[:, 2:2 + M, pad:pad + N] = 123.0
    assert torch.all(buf == 123.0)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 64, 300])
def test_any_matrix_scale(ctx, M):
    """nvfp4 with matrix scales that are not powers of two, as other programs write them."""
    A, B = _mx(ctx, (2, M, 320), 9, "nvfp4"), _mx(ctx, (2, 200, 320), 10, "nvfp4")
    one = torch.ones(2, device="cuda")
    A1, B1 = A._replace(scale=one), B._replace(scale=one)
    D = ctx.defl_mx4_gemm(A._replace(scale=one * 0.3), B._replace(scale=one * 7.7), out_dtype=F32)
    _check(ctx, D, A1, B1, scale=float(np.float32(0.3)) * float(np.float32(7.7)))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shape", [(4, 200, 64), (64, 200, 320), (300, 200, 64), (16, 40, 4096)])
def test_scales_that_leave_fp32_together(ctx, fmt, shape):
    """Values near 2^83 on both sides: a sum of zeros is zero. nvfp4 forms its sums before the matrices' scales meet them: what is
    not zero is infinite with its sign, and values near 2^-93 and 2^-67 with an alpha of 2^100 give ordinary numbers. (mxfp4 has no
    scale of a matrix: there each product leaves fp32 by itself.) Factors are powers of two, so that the codes stay the same."""
    M, N, K = shape
    a, w = _rand((1, M, K), 13, F32, 0.0).cuda(), _rand((1, N, K), 14, F32, 0.0).cuda()
    a[0, 1], a[0, 2, 1:], w[0, 5] = 0.0, 0.0, 0.0
    a[0, 2, 0], w[0, :, 0] = 3.0, 0.0
    D = ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(a * 2.0 ** 83, fmt), ctx.defl_mx4_quantize(w * 2.0 ** 83, fmt), out_dtype=F32)
    zero = torch.zeros_like(D, dtype=torch.bool)
    zero[0, 1], zero[0, 2], zero[0, :, 5] = True, True, True
    assert torch.all(D[zero] == 0)
    if fmt == "nvfp4":
        plain = ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(a, fmt), ctx.defl_mx4_quantize(w, fmt), out_dtype=F32)
        large = plain != 0
        assert torch.all(D[large] == plain[large] * float("inf"))
        A, B = ctx.defl_mx4_quantize(a * 2.0 ** -93, fmt), ctx.defl_mx4_quantize(w * 2.0 ** -67, fmt)
        _check(ctx, ctx.defl_mx4_gemm(A, B, out_dtype=F32, alpha=2.0 ** 100), A, B, 2.0 ** 100)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [8, 64, 300])
def test_not_finite(ctx, fmt, M):
    """A block that is not finite makes NaN of its row (A) or column (B) of the product and of nothing else."""
    a, w = _rand((1, M, 200), 11, F32).cuda(), _rand((1, 90, 200), 12, F32).cuda()
    a[0, 3, 77], w[0, 50, 199] = float("inf"), float("nan")
    D = ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(a, fmt), ctx.defl_mx4_quantize(w, fmt))
    bad = torch.zeros_like(D, dtype=torch.bool)
    bad[0, 3], bad[0, :, 50] = True, True
    assert torch.equal(torch.isnan(D), bad) and torch.isfinite(D[~bad]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shape", [(300, 192, 320), (64, 70, 45), (5, 100, 33)])
def test_linear_layer_forward_and_backward(ctx, fmt, shape):
    """y, dx and dw of a linear layer against the formulas on the rounded matrices."""
    t, k, n = shape
    x, w, dy = _rand((1, t, k), 13, BF16).cuda(), _rand((1, n, k), 14, BF16).cuda(), _rand((1, t, n), 15, BF16).cuda()
    (xq, xt), (wq, wt), (gq, gt) = (ctx.defl_mx4_quantize(v, fmt, both=True) for v in (x, w, dy))
    _check(ctx, ctx.defl_mx4_gemm(xq, wq), xq, wq)
    _check(ctx, ctx.defl_mx4_gemm(gq, wt), gq, wt)
    _check(ctx, ctx.defl_mx4_gemm(gt, xt, out_dtype=F32), gt, xt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
def test_gradients_against_differences(ctx, fmt):
    """On matrices that both directions hold exactly (grid values, a six in every block) the rounding is the identity, L = sum(dy * y) is
    bilinear and a difference quotient of any step is its derivative: it has to be what the backward products give, exactly."""
    rng = np.random.default_rng(16)
    t, k, n = 160, 96, 64

    def make(rows, cols):
        x = rng.choice(np.concatenate([mx4.GRID, -mx4.GRID]), (1, rows, cols))
        x[:, ::16, ::16] = 6.0
        x[:, :, ::16], x[:, ::16, :] = 6.0, 6.0
        return torch.tensor(x, dtype=F32).cuda()
    x, w, dy = make(t, k), make(n, k), make(t, n)

    def loss(x, w):
        return float((dy.double() * ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(x, fmt), ctx.defl_mx4_quantize(w, fmt), out_dtype=F32).double()).sum())
    xt, wt = ctx.defl_mx4_quantize(x, fmt, transposed=True), ctx.defl_mx4_quantize(w, fmt, transposed=True)
    dq, dt = ctx.defl_mx4_quantize(dy, fmt, both=True)
    dx, dw = ctx.defl_mx4_gemm(dq, wt, out_dtype=F32), ctx.defl_mx4_gemm(dt, xt, out_dtype=F32)
    base = loss(x, w)
    for i, j in ((1, 1), (17, 40), (63, 95)):                # places without a six: the step goes to another grid value
        for m, grad, f in ((x, dx, lambda v: loss(v, w)), (w, dw, lambda v: loss(x, v))):
            v = m.clone()
            step = 3.0 if float(m[0, i, j]) < 3.0 and float(m[0, i, j]) in (-3.0, 0.0, 1.0) else -float(m[0, i, j]) if float(m[0, i, j]) else 2.0
            v[0, i, j] += step
            assert (f(v) - base) / step == float(grad[0, i, j])


@pytest.mark.gpu
def test_captured_and_on_two_streams(ctx):
    """A forward pass in two graphs of one context, replayed on two streams at once with new data in the inputs."""
    def call(x, w):
        return ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(x, "nvfp4"), ctx.defl_mx4_quantize(w, "nvfp4"))
    w = _rand((1, 500, 640), 17, BF16).cuda()
    xs = [_rand((1, 400, 640), s, BF16).cuda() for s in (18, 19)]
    call(xs[0], w)
    graphs = []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = call(x, w)
        graphs.append((g, y, torch.cuda.Stream()))
    for s in (20, 21):
        for x, d in zip(xs, (0, 2)):
            x.copy_(_rand((1, 400, 640), s + d, BF16))
        torch.cuda.synchronize()
        for g, _, st in graphs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for x, (_, y, _) in zip(xs, graphs):
            assert torch.equal(y, call(x, w))
    assert ctx.defl_device_wait_status() == 0


@pytest.mark.gpu
def test_offsets_past_32_bits(ctx):
    """Inputs, codes and results of more than 2^32 elements (and codes of more than 2^32 bytes): their last rows are right."""
    rows, cols = 132000, 65536
    part = _rand((1, 1000, cols), 22, BF16).cuda()
    X = part.expand(132, 1000, cols).reshape(1, rows, cols)
    q = ctx.defl_mx4_quantize(X, "mxfp4")
    del X
    want = ctx.defl_mx4_quantize(part, "mxfp4")
    assert q.codes.numel() > 2 ** 32 and torch.equal(q.codes[0, -1000:], want.codes[0])
    D = ctx.defl_mx4_dequantize(q)
    assert torch.equal(D[0, -1000:], ctx.defl_mx4_dequantize(want)[0])
    del q, D
    torch.cuda.empty_cache()
    A, B = _mx(ctx, (1, 66000, 64), 23, "mxfp4"), _mx(ctx, (1, 65600, 64), 24, "mxfp4")
    D = ctx.defl_mx4_gemm(A, B)
    # the same rows in a product of their own (a multiple of the tile further up: the same sums)
    tail = ctx.defl_mx4_quantize(_rand((1, 66000, 64), 23, F32)[:, -464:].contiguous().cuda(), "mxfp4")
    assert D.numel() > 2 ** 32 and torch.equal(D[0, -464:], ctx.defl_mx4_gemm(tail, B)[0])


@pytest.mark.gpu
def test_refusals(ctx):
    from paper_2609_21102_b200 import binding
    x = torch.randn(1, 64, 64, device="cuda")
    q = ctx.defl_mx4_quantize(x, "mxfp4")
    for bad in (x[0], x.half(), x.cpu(), x[:, ::2, ::2], x[:, :1].expand(1, 64, 64)):
        with pytest.raises(ValueError):
            ctx.defl_mx4_quantize(bad)
    with pytest.raises(ValueError):
        ctx.defl_mx4_quantize(x, "fp4")
    for bad in (q._replace(cols=96), q._replace(rows=200), q._replace(codes=q.codes.float()), q._replace(fmt="nvfp4"), q._replace(fmt="e2m1"),
                q._replace(scales=q.scales[:, :, :, :256])):
        with pytest.raises(ValueError):
            ctx.defl_mx4_dequantize(bad)
        with pytest.raises(ValueError):
            ctx.defl_mx4_gemm(q, bad)
    with pytest.raises(ValueError):
        ctx.defl_mx4_gemm(q, ctx.defl_mx4_quantize(x, "nvfp4"))
    with pytest.raises(ValueError):
        ctx.defl_mx4_gemm(q, ctx.defl_mx4_quantize(x[:, :, :32], "mxfp4"))
    with pytest.raises(ValueError):
        ctx.defl_mx4_gemm(q, ctx.defl_mx4_quantize(x.expand(3, 64, 64).contiguous(), "mxfp4"))
    for out in (torch.empty(1, 64, 63, device="cuda"), torch.empty(1, 64, 64), torch.empty(1, 64, 64, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            ctx.defl_mx4_gemm(q, q, out=out)
    with pytest.raises(binding.DeflError) as e:
        ctx.defl_mx4_gemm(q, q, out_dtype=torch.float16)
    assert e.value.code == -1
    with pytest.raises(binding.DeflError):
        ctx.defl_mx4_dequantize(q, torch.float16)
    with pytest.raises(binding.DeflError):                   # rows of the result that overlap
        ctx.defl_mx4_gemm(q, q, out=torch.empty(64, device="cuda").expand(1, 64, 64))
    with pytest.raises(binding.DeflError):
        ctx.defl_mx4_quantize(torch.empty(1, 0, 64, device="cuda"))


def test_refusals_and_sizes_without_a_device():
    import ctypes
    from paper_2609_21102_b200 import binding, build
    build.build()
    L = binding.lib()
    with pytest.raises(ValueError):
        binding._native().mx4_quantize(0, 0, torch.zeros(1, 4, 4), "mxfp4", 1, binding.Mx4)
    with pytest.raises(ValueError):
        binding._native().mx4_quantize(0, 0, torch.zeros(1, 4, 4), "fp4", 1, binding.Mx4)
    with pytest.raises(TypeError):
        binding._native().mx4_quantize(0, 0, None, "nvfp4", 1, binding.Mx4)
    assert L.defl_mx4_quantize(None, None, 0, 1, 1, 1, ctypes.c_int64(1), ctypes.c_int64(1), 0, None, None, None) == -1
    assert L.defl_mx4_dequantize(None, None, 1, 1, 1, 0, None, 0) == -1
    assert L.defl_mx4_gemm(None, None, None, 1, 1, 1, 1, 0, 0, ctypes.c_float(1.0), None, ctypes.c_int64(1), ctypes.c_int64(1), 0, None) == -1
    assert L.defl_mx4_gemm_work_bytes(None, 1, 128, 64, 6400, 0) == 0
    for b, rows, cols in ((1, 1, 1), (2, 129, 33), (3, 128, 64), (1, 517, 1003)):
        for fmt, code in binding.MX4_FORMATS.items():
            # every block of a matrix has a byte in its tiles
            index, byte, _ = mx4.quantize(np.ones((rows, cols)), fmt)
            assert L.defl_mx4_codes_bytes(b, rows, cols) == b * index.size // 2 == b * rows * -(-cols // 32) * 16
            assert L.defl_mx4_scales_bytes(b, rows, cols, code) == b * mx4.tiles(byte).size
    assert L.defl_mx4_codes_bytes(0, 1, 1) == 0 and L.defl_mx4_scales_bytes(1, 1, 1, 7) == 0 and L.defl_mx4_work_bytes(0) == 0
    assert L.defl_mx4_work_bytes(1) == 592 * 4 and L.defl_mx4_work_bytes(1000) == 4000


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shape", [(1, 64, 64, 64), (1, 300, 256, 512), (2, 700, 600, 4000), (1, 9, 7, 2300)])
def test_bounded_wait_runs_out_and_is_reported(monkeypatch, ctx, fmt, shape):
    """A wait that nothing satisfies ends in a status bit and a normal return: no codes are announced or copied, with the
    limit at 2 ms (one CTA a tile, pairs, several tiles a pair, parts along K). What was asked for has landed long
    before the waits give up; the word stays until it is cleared and the context stays usable."""
    from paper_2609_21102_b200 import binding
    b, M, N, K = shape
    A, B = _mx(ctx, (b, M, K), 31, fmt), _mx(ctx, (b, N, K), 32, fmt)
    few = A._replace(codes=A.codes[:, :1].contiguous(), scales=A.scales[:, :1].contiguous(), rows=1)
    torch.cuda.synchronize()
    monkeypatch.setenv("DEFL_MX4_HOLD", "1")
    monkeypatch.setenv("DEFL_TC_WAIT_MS", "2")
    held = binding.Context(0)
    assert held.defl_device_wait_status() == 0
    held.defl_mx4_gemm(A, B)
    assert held.defl_device_wait_status(clear=False) == binding.ST_DEVICE_WAIT
    assert held.defl_device_wait_status() == binding.ST_DEVICE_WAIT and held.defl_device_wait_status() == 0
    _check(held, held.defl_mx4_gemm(few, B, out_dtype=F32), few, B)            # (a single row waits for nothing)
    assert held.defl_device_wait_status() == 0
    held.close()
    _check(ctx, ctx.defl_mx4_gemm(A, B, out_dtype=F32), A, B)
    assert ctx.defl_device_wait_status() == 0


@pytest.mark.gpu
def test_wait_that_ran_out_is_not_lost_in_a_later_call(monkeypatch):
    """The order of a training step on one context: a 4-bit product whose wait runs out, then calls that clear and report a wait word of
    their own. The product's bit is still there, and is nobody else's."""
    from paper_2609_21102_b200 import binding
    monkeypatch.setenv("DEFL_MX4_HOLD", "1")
    monkeypatch.setenv("DEFL_TC_WAIT_MS", "50")
    held = binding.Context(0)
    A, B = _mx(held, (1, 300, 256), 33, "nvfp4"), _mx(held, (1, 128, 256), 34, "nvfp4")
    G = torch.tensor(np.random.default_rng(35).standard_normal((2, 128, 256))).float().cuda()
    sched = [list(binding.MUON_QUINTIC)] * 5
    held.defl_mx4_gemm(A, B)
    _, info = held.defl_polar_batched(G.bfloat16(), 4, 4, 1, sched, seed=1, want_info=True)
    held.defl_muon_step_batched(G.clone(), G.clone(), G, 0.02, 0.9, 4, 4, 1, sched)
    held.defl_psd_project((G[0, :, :128] + G[0, :, :128].T).contiguous(), 0, torch.eye(128, device="cuda")[:, :4].contiguous(), [list(binding.CLASSICAL_QUINTIC)] * 3)
    assert info["status"].cpu().tolist() == [0, 0]
    assert held.defl_device_wait_status(clear=False) == binding.ST_DEVICE_WAIT
    assert held.defl_device_wait_status() == binding.ST_DEVICE_WAIT and held.defl_device_wait_status() == 0
    held.close()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("shape", [(1, 5, 37), (2, 37, 130), (1, 200, 257)])
def test_padding_of_a_block_that_is_not_finite(ctx, fmt, dtype, bad, shape):
    """Columns (and for the transpose rows) that do not exist are zeros beside a value that is not finite too, by either way in."""
    X = _rand(shape, 36, dtype)
    X[0, 1, -1], X[0, -1, 2] = bad, bad
    for part in (X.cuda(), torch.nn.functional.pad(X, (0, 7)).cuda()[:, :, :-7]):
        q, qt = ctx.defl_mx4_quantize(part, fmt, both=True)
        P = part.double().cpu().numpy()
        _same(q, P, fmt)
        _same(qt, P.transpose(0, 2, 1), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 3, 8, 9, 200])
@pytest.mark.parametrize("up", [120, 100, -120])
def test_mxfp4_rows_far_apart_in_size(ctx, rows, up):
    """A near 2^up and B near 2^-up: a block's sum times one of its two scales may leave fp32 (32 products of at least 9 times 2^120), times
    both it is an ordinary number. Grid values with a six in every block: the sums are exact and so is the result."""
    rng = np.random.default_rng(37)

    def make(n):
        x = rng.choice([3.0, 4.0, 6.0], (1, n, 352))
        x[:, :, ::32] = 6.0
        return torch.tensor(x, dtype=F32).cuda()
    a, w = make(rows), make(90)
    A, B = ctx.defl_mx4_quantize(a * 2.0 ** up, "mxfp4"), ctx.defl_mx4_quantize(w * 2.0 ** -up, "mxfp4")
    want = a.double() @ w.double().transpose(1, 2)
    assert torch.equal(ctx.defl_mx4_gemm(A, B, out_dtype=F32).double(), want)
    assert torch.equal(ctx.defl_mx4_gemm(B, A, out_dtype=F32).double(), want.transpose(1, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shape", [(1, 1, 16384, 96), (1, 1, 16385, 96), (1, 2, 8193, 2048), (1, 8, 2048, 2048), (1, 8, 2049, 2048), (1, 3, 9000, 1600),
                                   (3, 5, 6000, 500), (40, 1, 410, 64), (1, 4, 700, 1000), (1, 7, 600, 1056), (1, 2, 890, 1056)])
def test_few_rows_in_either_form(ctx, fmt, shape):
    """Both sides of the rules that choose between the row kernel and the tensor cores, and its lanes: grid values with a six in every block, whose
    sums are exact in any order (a multiple of 1/4 below 36 K < 2^22), and values of any size against fp64."""
    b, M, N, K = shape
    rng = np.random.default_rng(39)
    vals = np.concatenate([mx4.GRID, -mx4.GRID])

    def make(rows):
        x = rng.choice(vals, (b, rows, K))
        x[:, :, ::16] = 6.0
        return torch.tensor(x, dtype=F32).cuda()
    a, w = make(M), make(N)
    D = ctx.defl_mx4_gemm(ctx.defl_mx4_quantize(a, fmt), ctx.defl_mx4_quantize(w, fmt), out_dtype=F32)
    assert torch.equal(D.double(), a.double() @ w.double().transpose(1, 2))
    A, B = _mx(ctx, (b, M, K), 40, fmt), _mx(ctx, (b, N, K), 41, fmt)
    _check(ctx, ctx.defl_mx4_gemm(A, B), A, B)
    assert ctx.defl_device_wait_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float64, torch.float16, torch.int8, torch.float8_e4m3fn, None])
def test_result_types_that_there_are_not(ctx, dtype):
    """All are refused as arguments, those that the library has no number for too."""
    from paper_2609_21102_b200 import binding
    q = ctx.defl_mx4_quantize(torch.ones(1, 4, 32, device="cuda"))
    for call in (lambda: ctx.defl_mx4_dequantize(q, dtype), lambda: ctx.defl_mx4_gemm(q, q, out_dtype=dtype)):
        with pytest.raises(binding.DeflError) as e:
            call()
        assert e.value.code == -1
