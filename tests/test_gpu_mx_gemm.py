"""Products of two microscaled 4-bit matrices on the tensor cores, against float64."""
import numpy as np
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    ctx = P.Context(2, 2, device=0)
    yield ctx
    assert P.llvq_last_error(ctx) == (0, 0)              # no wait ran out


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run(P, ctx, tokens, n_out, k_in, x=None, w=None, **kw):
    x, w = x or mx.random_matrix(tokens, k_in, seed=tokens, lo=120, hi=134), w or mx.random_matrix(n_out, k_in, seed=n_out + k_in)
    y = P.llvq_mx_gemm(ctx, dev(x[0]), dev(x[1]), tokens, dev(w[0]), dev(w[1]), n_out, k_in, **kw)
    return y, mx.values_of(*x, k_in), mx.values_of(*w, k_in)


def check(y, x, w):
    """The products are exact; a step of 64 columns is added to the running sum with at most four truncations (its two blocks, their sum, the
    running sum) of 2^-23 of what they add up, and the result takes half a step of bf16 on top."""
    got, want, size = y.double().cpu().numpy(), x @ w.T, np.abs(x) @ np.abs(w).T
    slack = 4 * (x.shape[1] / 64 + 1) * 2.0 ** -23 * size
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    assert (np.abs(got - want)[fine] <= (slack + 2.0 ** -8 * (np.abs(want) + slack))[fine]).all()


@pytest.mark.parametrize("tokens,n_out,k_in", [(1, 1, 1), (1, 128, 64), (64, 128, 256), (3, 5, 31), (65, 129, 257), (64, 128, 512), (100, 300, 480), (7, 1000, 1100),
                                               (200, 384, 4104), (33, 70, 9001)])
def test_product(P, ctx, tokens, n_out, k_in):
    y, x, w = run(P, ctx, tokens, n_out, k_in)
    assert y.dtype == torch.bfloat16 and tuple(y.shape) == (tokens, n_out)
    check(y, x, w)


@pytest.mark.parametrize("tokens,n_out,k_in", [(2017, 4300, 1300), (1000, 10000, 320), (448, 9472, 2080), (128, 19000, 288), (300, 18943, 256), (3000, 2000, 96), (2600, 4100, 544), (129, 20001, 1056)])
def test_several_tiles_per_thread_block(P, ctx, tokens, n_out, k_in):
    y, x, w = run(P, ctx, tokens, n_out, k_in)
    check(y, x, w)


def test_single_elements_meet_their_own_scales(P, ctx):
    # one non-zero block per row: every pair of (row, block) positions is told apart by its scales
    k_in, rows = 1024, 256
    g = np.random.default_rng(5)
    codes = np.zeros((rows, k_in // 2), dtype=np.uint8)
    scales = np.full((rows, mx.pitch(k_in)), 127, dtype=np.uint8)
    scales[:, :32] = g.integers(110, 140, (rows, 32))
    for r in range(rows):
        b = r % 32
        codes[r, 16 * b:16 * b + 16] = g.integers(0, 256, 16)
    ones = np.full((rows, k_in // 2), 0x22, dtype=np.uint8)
    other = np.full_like(scales, 127)
    for x, w in (((codes, scales), (ones, other)), ((ones, other), (codes, scales)), ((codes, scales), (codes, scales))):
        y, xv, wv = run(P, ctx, rows, rows, k_in, x, w)
        check(y, xv, wv)


@pytest.mark.parametrize("side", ["x", "w"])
def test_a_block_that_is_nan_reaches_its_row_alone(P, ctx, side):
    x, w = mx.random_matrix(70, 480, seed=1, lo=120, hi=134), mx.random_matrix(150, 480, seed=2)
    (x if side == "x" else w)[1][66, 14] = 255
    y, xv, wv = run(P, ctx, 70, 150, 480, x, w)
    check(y, xv, wv)
    assert torch.isnan(y).sum() == (150 if side == "x" else 70)


@pytest.mark.parametrize("xs,ws", [(1, 250), (250, 1), (60, 190), (127, 127)])
def test_far_scales_that_meet_in_the_middle(P, ctx, xs, ws):
    y, x, w = run(P, ctx, 40, 200, 320, mx.random_matrix(40, 320, seed=1, lo=xs, hi=xs + 3), mx.random_matrix(200, 320, seed=2, lo=ws, hi=ws + 2))
    check(y, x, w)


def test_writes_its_result_alone_and_the_same_every_time(P, ctx):
    tokens, n_out, k_in = 131, 333, 1000
    buf = torch.full((tokens * n_out + 10,), 4.0, dtype=torch.bfloat16, device="cuda")
    y, x, w = run(P, ctx, tokens, n_out, k_in, d_y=buf[5:-5])
    check(buf[5:-5].view(tokens, n_out), x, w)
    assert (buf[:5] == 4).all() and (buf[-5:] == 4).all()
    again, _, _ = run(P, ctx, tokens, n_out, k_in)
    assert torch.equal(again.view(-1), buf[5:-5])


def test_nothing_to_do(P, ctx):
    none = torch.empty((0, 32), dtype=torch.uint8, device="cuda")
    c, s = (dev(a) for a in mx.random_matrix(4, 64, seed=1))
    assert tuple(P.llvq_mx_gemm(ctx, none, none, 0, c, s, 4, 64).shape) == (0, 4)
    assert tuple(P.llvq_mx_gemm(ctx, c, s, 4, none, none, 0, 64).shape) == (4, 0)
    assert (P.llvq_mx_gemm(ctx, none, none, 3, none, none, 4, 0) == 0).all()
    with pytest.raises(P.LlvqError) as e:
        P.llvq_mx_gemm(ctx, c.view(-1)[1:97], s, 3, c, s, 4, 64)
    assert e.value.status == 2


def test_quantized_prompt_captured_and_on_two_streams(P, ctx):
    x, w = torch.randn((150, 1024), device="cuda").bfloat16(), torch.randn((640, 1024), device="cuda")
    wc, ws = P.llvq_mx_quantize(ctx, w)
    xc, xs = P.llvq_mx_quantize(ctx, x)
    want = P.llvq_mx_gemm(ctx, xc, xs, 150, wc, ws, 640, 1024)
    check(want, P.llvq_mx_dequant_matrix(ctx, xc, xs, 150, 1024).double().cpu().numpy(), P.llvq_mx_dequant_matrix(ctx, wc, ws, 640, 1024).double().cpu().numpy())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y1 = torch.empty_like(want)
    P.llvq_mx_gemm(ctx, xc, xs, 150, wc, ws, 640, 1024, y1, stream=side)
    y2 = P.llvq_mx_gemm(ctx, xc, xs, 150, wc, ws, 640, 1024)
    side.synchronize()
    assert torch.equal(y1, want) and torch.equal(y2, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, s = P.llvq_mx_quantize(ctx, x)
        y = P.llvq_mx_gemm(ctx, c, s, 150, wc, ws, 640, 1024)
    x.mul_(4)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, 4 * want)
