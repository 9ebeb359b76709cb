"""Products of 4-bit matrices with activations that are not finite: what the products and sums of binary32 give, however many there are."""
import numpy as np
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    ctx = P.Context(2, 2, device=0)
    yield ctx
    assert P.llvq_last_error(ctx) == (0, 0)              # no wait ran out


def expected(x, w):
    """For rows of X with an infinity: +inf, -inf, or NaN where an infinity meets zero or NaN, or both signs come; exact, as counts below 2^24 are in
    binary32.  None of it for other rows: NaN where either side has one, else 0 in place of the sum."""
    f = torch.float32
    up, down = (x == INF).to(f), (x == -INF).to(f)
    plus, minus = up @ (w > 0).to(f).T + down @ (w < 0).to(f).T, up @ (w < 0).to(f).T + down @ (w > 0).to(f).T
    zero = (up + down) @ (w == 0).to(f).T
    nan = torch.isnan(x).any(1)[:, None] | torch.isnan(w).any(1)[None] | (zero > 0) | ((plus > 0) & (minus > 0))
    y = torch.where(plus > 0, INF, torch.where(minus > 0, -INF, 0.0))
    return torch.where(nan, NAN, y)


def check(y, x, w):
    want, y = expected(x, w), y.float()
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    there = torch.isinf(want)
    assert torch.equal(y[there], want[there]) and torch.isfinite(y[~there & ~torch.isnan(want)]).all()


@pytest.mark.parametrize("kind", ["one sign", "any weight"])
def test_rows_full_of_infinities_on_a_matrix_of_several_tiles_per_thread_block(P, ctx, kind):
    # 501 tiles of 256 rows: three or four for each of 148 thread blocks.  Rows of W of one sign without a zero are looked through to the end.
    n_out, k_in, batch = 128256, 2048, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    low = torch.randint(1 if kind == "one sign" else 0, 8, (2, n_out, k_in // 2), generator=g, device="cuda", dtype=torch.uint8)
    sign = torch.randint(0, 2, (n_out, 1) if kind == "one sign" else (2, n_out, k_in // 2), generator=g, device="cuda", dtype=torch.uint8) * 8
    codes = (low + sign)[0] | (low + sign)[1] << 4
    scales = torch.full((n_out, mx.pitch(k_in)), 120, dtype=torch.uint8, device="cuda")
    w = P.llvq_mx_dequant_matrix(ctx, codes, scales, n_out, k_in)
    x = torch.full((batch, k_in), INF, device="cuda").bfloat16()
    x[1] = -INF
    x[2, :-1] = 1.0                                       # the last column alone
    x[3] = 1.0                                            # none
    for _ in range(3):
        y = P.llvq_mx_gemm_small_batch(ctx, codes, scales, n_out, k_in, x)
    check(y, x, w)
    if kind == "one sign":
        assert torch.isinf(y).sum() == 63 * n_out
    assert P.llvq_last_error(ctx) == (0, 0)


@pytest.mark.parametrize("batch", [2, 16, 17, 40, 64])
@pytest.mark.parametrize("n_out,k_in", [(40, 33), (300, 1001), (5000, 2500)])
def test_infinities_and_nan_here_and_there(P, ctx, n_out, k_in, batch):
    codes, scales = mx.random_matrix(n_out, k_in, seed=n_out)
    g = np.random.default_rng(batch)
    codes[n_out // 2:] |= 0x11                            # half of the rows without a zero
    if k_in % 32:
        codes[:, (k_in + 1) // 2:] = 0
        if k_in % 2:
            codes[:, k_in // 2] &= 15
    scales[3, 0] = 255
    scales[n_out - 1, mx.blocks(k_in) - 1] = 255
    w = torch.from_numpy(mx.values_of(codes, scales, k_in)).float().cuda()
    x = torch.randn((batch, k_in), generator=torch.Generator().manual_seed(batch))
    for n in range(batch):
        kind = n % 5
        where = g.choice(k_in, size=min(k_in, 1 + n % 3), replace=False)
        if kind == 1:
            x[n, where[0]] = INF
        elif kind == 2:
            x[n, where] = -INF
        elif kind == 3:
            x[n, where] = INF
            x[n, int(g.integers(k_in))] = NAN
        elif kind == 4:
            x[n, k_in - 1] = -INF if n % 2 else INF
    x = x.bfloat16().cuda()
    y = P.llvq_mx_gemm_small_batch(ctx, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), n_out, k_in, x)
    check(y, x, w)
    assert P.llvq_last_error(ctx) == (0, 0)

@pytest.mark.parametrize("batch", [1, 3, 8, 16])
@pytest.mark.parametrize("others", [0.0, 2.0 ** -133, 2.0 ** -126])
@pytest.mark.parametrize("scale", [0, 1, 2, 254])
def test_an_infinity_among_zeros_meets_the_smallest_scales(P, ctx, batch, others, scale):
    # columns 0 to 511 of X hold nothing else, or the smallest numbers there are: the smallest scale is 2^-127, and times an infinity it is one
    n_out, k_in = 40, 520
    codes, scales = mx.random_matrix(n_out, k_in, seed=3)
    codes[:20] |= 0x11
    codes[:, k_in // 2:] = 0
    scales[:, :16] = scale
    w = torch.from_numpy(mx.values_of(codes, scales, k_in)).float().cuda()
    x = torch.full((batch, k_in), others)
    x[0, 77] = INF
    x[batch - 1, 200] = -INF
    x = x.bfloat16().cuda()
    codes, scales = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    check(P.llvq_mx_gemm_small_batch(ctx, codes, scales, n_out, k_in, x), x, w)
    check(P.llvq_mx_gemv(ctx, codes, scales, n_out, k_in, x[0])[None], x[:1], w)
