"""Quantisation to microscaled 4-bit floating point and products with such matrices, against float64."""
import numpy as np
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    return P.Context(2, 2, device=0)


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def f64(t):
    return t.detach().double().cpu().numpy()


def check_product(y, x, w):
    """Products of bf16 numbers are exact in binary32.  128 columns are summed by eight tensor-core steps, each with a truncation of at most
    2^-23 of what it adds up, then the K / 128 partial sums and those of up to 8 warps with one rounding of 2^-24 each: together less than
    (8 + K / 256 + 4) 2^-23 of the sum of the magnitudes; doubled for the second-order terms.  Then half a step of the result's type."""
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    got = f64(y)
    slack = 2 * (12 + w.shape[1] / 256) * 2.0 ** -23 * size
    step = torch.finfo(y.dtype).eps / 2
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    assert (np.abs(got - want)[fine] <= (slack + step * (np.abs(want) + slack))[fine]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 31), (2, 33), (5, 256), (7, 520), (4, 513), (33, 4104), (257, 64)])
def test_quantize_and_back(P, ctx, dtype, rows, cols):
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = (torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, 1), generator=g))).to(DTYPES[dtype])
    x[torch.rand((rows, cols), generator=g) < 0.1] = 0
    codes, scales, values = mx.quantize(x.double().numpy())
    c, s = P.llvq_mx_quantize(ctx, x.cuda())
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scales)
    assert np.array_equal(f64(P.llvq_mx_dequant_matrix(ctx, c, s, rows, cols)), values)


def test_quantize_at_the_borders(P, ctx):
    # ties at every middle between two elements and just beside them, both signs; the largest of a block, what saturates, zeros, subnormals
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    near = [m * (1 + d) for m in mids for d in (-2.0 ** -20, 0.0, 2.0 ** -20)]
    rows = [near + [4.0] + [0.0] * 10, [-v for v in near] + [-7.99] + [-0.0] * 10, [0.0] * 32, [2.0 ** -149] * 32, [2.0 ** -126] + [2.0 ** -130] * 31,
            [2.0 ** -127] * 32, [3.0e38] + [1.0e37] * 31, [float("inf")] + [1.0] * 31, [float("nan")] + [1.0] * 31, [1.0] * 31 + [float("-inf")]]
    x = torch.tensor(rows, dtype=torch.float32)
    codes, scales, values = mx.quantize(x.double().numpy())
    c, s = P.llvq_mx_quantize(ctx, x.cuda())
    assert np.array_equal(s.cpu().numpy(), scales) and np.array_equal(c.cpu().numpy(), codes)
    back = f64(P.llvq_mx_dequant_matrix(ctx, c, s, 10, 32))
    assert np.array_equal(back, values, equal_nan=True) and np.isnan(back[7:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_a_larger_matrix_are_quantized_in_place(P, ctx, dtype):
    big = torch.randn((40, 777), device="cuda").to(DTYPES[dtype])
    for view in (big[3:30, 5:300], big[::2, :777], big[:, 8:40], big[:1, 1:778]):
        c, s = P.llvq_mx_quantize(ctx, view)
        d, t = P.llvq_mx_quantize(ctx, view.contiguous())
        assert torch.equal(c, d) and torch.equal(s, t)
    with pytest.raises(AssertionError):
        P.llvq_mx_quantize(ctx, big.T)
    with pytest.raises(AssertionError):
        P.llvq_mx_quantize(ctx, big[0].expand(4, 777))


@pytest.mark.parametrize("rows,cols,ld,shift", [(9, 40, 40, 0), (9, 41, 41, 0), (5, 511, 520, 0), (5, 513, 515, 3), (3, 7, 9, 1), (1, 1, 1, 5), (64, 4104, 4104, 4)])
def test_dequantize_into_part_of_a_buffer(P, ctx, rows, cols, ld, shift):
    codes, scales = mx.random_matrix(rows, cols, seed=cols, lo=0, hi=252)
    buf = torch.full((shift + rows * ld + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    P.llvq_mx_dequant_matrix(ctx, dev(codes), dev(scales), rows, cols, buf[shift:shift + (rows - 1) * ld + cols], ld)
    got = f64(buf)
    want = np.full(got.shape, 7.0)
    for r in range(rows):
        want[shift + r * ld:shift + r * ld + cols] = mx.values_of(codes, scales, cols)[r]
    assert np.array_equal(got, want)


@pytest.mark.parametrize("n_out,k_in", [(1, 1), (1, 32), (15, 33), (17, 480), (300, 512), (129, 1100), (64, 4096), (40, 4104), (33, 9001)])
@pytest.mark.parametrize("y_dtype", [torch.float32, torch.bfloat16])
def test_gemv(P, ctx, n_out, k_in, y_dtype):
    codes, scales = mx.random_matrix(n_out, k_in, seed=n_out + k_in)
    x = torch.randn(k_in, generator=torch.Generator().manual_seed(k_in)).bfloat16()
    y = P.llvq_mx_gemv(ctx, dev(codes), dev(scales), n_out, k_in, x.cuda(), y_dtype=y_dtype)
    assert y.dtype == y_dtype and tuple(y.shape) == (n_out,)
    check_product(y[None], f64(x)[None], mx.values_of(codes, scales, k_in))


@pytest.mark.parametrize("batch", [1, 2, 7, 8, 9, 16, 17, 31, 33, 63, 64])
@pytest.mark.parametrize("n_out,k_in", [(70, 256), (33, 1001), (48, 1002), (130, 1004)])
def test_small_batches(P, ctx, batch, n_out, k_in):
    codes, scales = mx.random_matrix(n_out, k_in, seed=n_out + k_in)
    x = torch.randn((batch, k_in), generator=torch.Generator().manual_seed(batch)).bfloat16()
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), n_out, k_in, x.cuda())
    assert y.dtype == torch.bfloat16 and tuple(y.shape) == (batch, n_out)
    check_product(y, f64(x), mx.values_of(codes, scales, k_in))


@pytest.mark.parametrize("batch", [1, 5, 17, 32, 33, 64])
@pytest.mark.parametrize("n_out,k_in", [(9000, 3850), (300, 12000), (2600, 13000)])
def test_larger_matrices(P, ctx, batch, n_out, k_in):
    # sizes at which thread blocks share tiles, take several of them, and change from one form of the product to the other
    codes, scales = mx.random_matrix(n_out, k_in, seed=n_out)
    x = torch.randn((batch, k_in), generator=torch.Generator().manual_seed(batch)).bfloat16()
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), n_out, k_in, x.cuda())
    check_product(y, f64(x), mx.values_of(codes, scales, k_in))


@pytest.mark.parametrize("batch", [1, 3, 20, 40])
def test_an_infinity_in_the_activations(P, ctx, batch):
    # +-inf where the weight is not zero, NaN where it is, as products in binary32 give; other rows as if it were not there
    codes, scales = mx.random_matrix(300, 480, seed=3)
    w = mx.values_of(codes, scales, 480)
    x = torch.randn((batch, 480), generator=torch.Generator().manual_seed(1)).bfloat16()
    clean = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 300, 480, x.cuda())
    x[0, 77] = float("inf")
    y = f64(P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 300, 480, x.cuda()))
    want = np.where(w[:, 77] == 0, np.nan, np.where(w[:, 77] < 0, -np.inf, np.inf))
    assert np.array_equal(y[0], want, equal_nan=True) and np.array_equal(y[1:], f64(clean)[1:])


@pytest.mark.parametrize("batch", [1, 3, 20, 40])
def test_activations_of_very_different_sizes(P, ctx, batch):
    # one channel 2^17 times the others, where every weight is zero: the others count as if it were not there (down to 2^-19 of the largest exactly)
    codes, scales = mx.random_matrix(64, 480, seed=3)
    codes[:, 50] = 0                                          # columns 100 and 101
    x = torch.randn((batch, 480), generator=torch.Generator().manual_seed(1)).bfloat16()
    x[:, 100] = 2.0 ** 17
    x[:, 101] = 0
    x = torch.where(x.abs() < 2.0 ** -2, torch.zeros_like(x), x)
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 64, 480, x.cuda())
    check_product(y, f64(x), mx.values_of(codes, scales, 480))


@pytest.mark.parametrize("batch", [1, 3, 16])
def test_activations_that_become_subnormal_binary16(P, ctx, batch):
    # one channel 2^28 to 2^30 times the others, where every weight is zero: up to 16 rows of X are exact down to 2^-32 of the largest
    codes, scales = mx.random_matrix(64, 480, seed=3)
    codes[:, 50] = 0                                          # columns 100 and 101
    x = torch.randn((batch, 480), generator=torch.Generator().manual_seed(1)).bfloat16()
    x = torch.where(x.abs() < 2.0 ** -2, torch.zeros_like(x), x)
    x[:, 100] = 2.0 ** 28
    x[:, 101] = 0
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 64, 480, x.cuda())
    check_product(y, f64(x), mx.values_of(codes, scales, 480))


@pytest.mark.parametrize("lo,hi", [(0, 3), (126, 130), (120, 200), (8, 240)])
def test_products_over_the_whole_range_of_scales(P, ctx, lo, hi):
    # activations that bring the products back into the middle of binary32's range
    n_out, k_in = 32, 1024
    codes, scales = mx.random_matrix(n_out, k_in, seed=lo, lo=lo, hi=hi)
    w = mx.values_of(codes, scales, k_in)
    x = torch.randn((40, k_in), generator=torch.Generator().manual_seed(1)) * 2.0 ** (122 - (lo + hi) // 2)
    x = x.bfloat16()
    y = P.llvq_mx_gemv(ctx, dev(codes), dev(scales), n_out, k_in, x[0].cuda())
    check_product(y[None], f64(x[:1]), w)
    for batch in (3, 20, 40):
        check_product(P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), n_out, k_in, x[:batch].cuda()), f64(x[:batch]), w)


def test_a_block_that_is_nan_reaches_its_row_alone(P, ctx):
    codes, scales = mx.random_matrix(40, 480, seed=3)
    scales[5, 14] = 255
    x = torch.randn((3, 480)).bfloat16()
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 40, 480, x.cuda())
    check_product(y, f64(x), mx.values_of(codes, scales, 480))
    assert torch.isnan(y[:, 5]).all() and torch.isnan(y).sum() == 3
    x = torch.randn((50, 480)).bfloat16()
    check_product(P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 40, 480, x.cuda()), f64(x), mx.values_of(codes, scales, 480))


def test_activations_that_are_not_finite_reach_their_own_row(P, ctx):
    codes, scales = mx.random_matrix(40, 480, seed=3)
    x = torch.randn((3, 480)).bfloat16()
    clean = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 40, 480, x.cuda())
    x[1, 100] = float("nan")
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 40, 480, x.cuda())
    assert torch.isnan(y[1]).all() and torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2])


@pytest.mark.parametrize("shift", [1, 2, 4])
def test_activations_off_the_16_byte_boundaries(P, ctx, shift):
    codes, scales = mx.random_matrix(40, 520, seed=3)
    buf = torch.randn(5 * 520 + 8).bfloat16().cuda()
    x = buf[shift:shift + 5 * 520].view(5, 520)
    y = P.llvq_mx_gemm_small_batch(ctx, dev(codes), dev(scales), 40, 520, x)
    check_product(y, f64(x), mx.values_of(codes, scales, 520))


def test_products_are_the_same_every_time_and_touch_nothing_else(P, ctx):
    codes, scales = (dev(a) for a in mx.random_matrix(1000, 4096, seed=3))
    for batch in (1, 7, 20, 50):
        x = torch.randn((batch, 4096), device="cuda").bfloat16()
        y = torch.full((batch * 1000 + 8,), 3.0, dtype=torch.bfloat16, device="cuda")
        P.llvq_mx_gemm_small_batch(ctx, codes, scales, 1000, 4096, x, y[4:-4])
        assert (y[:4] == 3).all() and (y[-4:] == 3).all()
        for _ in range(3):
            assert torch.equal(P.llvq_mx_gemm_small_batch(ctx, codes, scales, 1000, 4096, x).view(-1), y[4:-4])


@pytest.mark.parametrize("n_out,k_in,batch", [(10311, 8290, 20), (10311, 8290, 48), (20000, 4096, 64), (4096, 11004, 5), (11008, 4096, 1)])
def test_products_are_the_same_many_times(P, ctx, n_out, k_in, batch):
    # busy shared memory: a place that is given back before all lanes have read it showed in about one call of a hundred
    g = torch.Generator(device="cuda").manual_seed(5)
    codes = torch.randint(0, 256, (n_out, mx.blocks(k_in) * 16), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.randint(110, 125, (n_out, mx.pitch(k_in)), dtype=torch.uint8, device="cuda", generator=g)
    x = torch.randn((batch, k_in), device="cuda", generator=g).bfloat16()
    first = P.llvq_mx_gemm_small_batch(ctx, codes, scales, n_out, k_in, x)
    same = torch.ones((), dtype=torch.bool, device="cuda")
    for _ in range(400):
        same &= (P.llvq_mx_gemm_small_batch(ctx, codes, scales, n_out, k_in, x) == first).all()
    assert bool(same)


def test_nothing_to_do(P, ctx):
    none = torch.empty((0, 0), dtype=torch.uint8, device="cuda")
    c, s = P.llvq_mx_quantize(ctx, torch.empty((0, 64), device="cuda"))
    assert tuple(c.shape) == (0, 32) and tuple(s.shape) == (0, 16)
    assert tuple(P.llvq_mx_quantize(ctx, torch.empty((4, 0), device="cuda"))[0].shape) == (4, 0)
    assert P.llvq_mx_gemv(ctx, none, none, 0, 64, torch.zeros(64, device="cuda").bfloat16()).numel() == 0
    assert (P.llvq_mx_gemv(ctx, none, none, 5, 0, torch.zeros(0, device="cuda").bfloat16()) == 0).all()
    assert P.llvq_mx_gemm_small_batch(ctx, torch.zeros((4, 32), dtype=torch.uint8, device="cuda"), torch.zeros((4, 16), dtype=torch.uint8, device="cuda"), 4, 64,
                                      torch.zeros((0, 64), device="cuda").bfloat16()).numel() == 0


def test_misaligned_codes_are_refused(P, ctx):
    buf = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    x = torch.zeros(64, device="cuda").bfloat16()
    for f in (lambda: P.llvq_mx_gemv(ctx, buf[1:], buf, 4, 64, x), lambda: P.llvq_mx_gemv(ctx, buf, buf[8:], 4, 64, x),
              lambda: P.llvq_mx_dequant_matrix(ctx, buf[1:], buf, 4, 64), lambda: P.llvq_mx_quantize(ctx, torch.zeros((4, 64), device="cuda"), buf[1:], buf)):
        with pytest.raises(P.LlvqError) as e:
            f()
        assert e.value.status == 2


@pytest.mark.parametrize("batch", [16, 50])
def test_captured_and_on_another_stream(P, ctx, batch):
    x = torch.randn((batch, 1024), device="cuda").bfloat16()
    w = torch.randn((512, 1024), device="cuda")
    wc, ws = P.llvq_mx_quantize(ctx, w)
    y = P.llvq_mx_gemm_small_batch(ctx, wc, ws, 512, 1024, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2 = P.llvq_mx_gemm_small_batch(ctx, wc, ws, 512, 1024, x)
    y3 = torch.empty_like(y)
    P.llvq_mx_gemm_small_batch(ctx, wc, ws, 512, 1024, x, y3, stream=side)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(y, y3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, s = P.llvq_mx_quantize(ctx, w)
        y4 = P.llvq_mx_gemm_small_batch(ctx, c, s, 512, 1024, x)
        back = P.llvq_mx_dequant_matrix(ctx, c, s, 512, 1024)
    w.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y4, 2 * y) and torch.equal(back, 2 * P.llvq_mx_dequant_matrix(ctx, wc, ws, 512, 1024))
