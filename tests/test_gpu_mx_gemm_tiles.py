"""Products of two 4-bit matrices in every tile: against float64, with blocks that are NaN, into a buffer of their own, and many times over."""
import numpy as np
import pytest
import torch

import mx_gemm_sizes
import mx_util as mx

pytestmark = pytest.mark.gpu
CASES = [size for sizes in mx_gemm_sizes.TILES.values() for size in sizes]


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


def check(y, x, w):
    """The products are exact; a step of 64 columns is added to the running sum with at most four truncations (its two blocks, their sum, the
    running sum) of 2^-23 of what they add up, and the result takes half a step of bf16 on top."""
    got, want, size = y.double(), x @ w.T, x.abs() @ w.abs().T
    slack = 4 * (x.shape[1] / 64 + 1) * 2.0 ** -23 * size
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert ((got - want).abs() <= slack + 2.0 ** -8 * (want.abs() + slack)).logical_or(torch.isnan(want)).all()


@pytest.mark.parametrize("tokens,n_out,k_in", CASES)
def test_product_in_every_tile(P, ctx, tokens, n_out, k_in):
    x, w = mx.random_matrix(tokens, k_in, seed=tokens, lo=120, hi=134), mx.random_matrix(n_out, k_in, seed=n_out + k_in)
    buf = torch.full((tokens * n_out + 16,), 4.0, dtype=torch.bfloat16, device="cuda")
    y = buf[8:-8].view(tokens, n_out)
    xv, wv = dev(mx.values_of(*x, k_in)), dev(mx.values_of(*w, k_in))
    P.llvq_mx_gemm(ctx, dev(x[0]), dev(x[1]), tokens, dev(w[0]), dev(w[1]), n_out, k_in, y)
    check(y, xv, wv)
    assert (buf[:8] == 4).all() and (buf[-8:] == 4).all()
    # a NaN block in the first, a middle and the last row of either side, in the first, a middle and the last block: those rows and columns alone
    g, clean = np.random.default_rng(1), y.clone()
    rows, cols = {0, int(g.integers(tokens)), tokens - 1}, {0, int(g.integers(n_out)), n_out - 1}
    for side, some in ((x, rows), (w, cols)):
        for i, r in enumerate(sorted(some)):
            side[1][r, (0, mx.blocks(k_in) // 2, mx.blocks(k_in) - 1)[i]] = 255
    y = P.llvq_mx_gemm(ctx, dev(x[0]), dev(x[1]), tokens, dev(w[0]), dev(w[1]), n_out, k_in)
    nan = torch.zeros((tokens, n_out), dtype=torch.bool, device="cuda")
    nan[sorted(rows)] = True
    nan[:, sorted(cols)] = True
    assert torch.equal(torch.isnan(y), nan) and torch.equal(y[~nan], clean[~nan])


@pytest.mark.parametrize("tokens,n_out,k_in", CASES)
def test_the_same_many_times(P, ctx, tokens, n_out, k_in):
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = [(torch.randint(0, 256, (n, mx.blocks(k_in) * 16), dtype=torch.uint8, device="cuda", generator=g),
             torch.randint(110, 125, (n, mx.pitch(k_in)), dtype=torch.uint8, device="cuda", generator=g)) for n in (tokens, n_out)]
    first = P.llvq_mx_gemm(ctx, *x, tokens, *w, n_out, k_in)
    same = torch.ones((), dtype=torch.bool, device="cuda")
    y = torch.empty_like(first)
    for _ in range(300):
        P.llvq_mx_gemm(ctx, *x, tokens, *w, n_out, k_in, y)
        same &= (y == first).all()
    assert bool(same)
