"""What products of 4-bit matrices promise of each activation: exact down to 2^-19 of the largest of its 32 columns, off by at most 2^-27 of that one below,
whatever other columns hold.  W is the unit matrix, so Y shows every activation by itself."""
import numpy as np
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu
K = 1100                                                  # three chunks of 512 columns, the last block ragged
BATCHES = [1, 2, 7, 8, 9, 16, 17, 32, 33, 64]


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    ctx = P.Context(2, 2, device=0)
    yield ctx
    assert P.llvq_last_error(ctx) == (0, 0)


@pytest.fixture(scope="module")
def unit():
    codes, scales = np.zeros((K, mx.blocks(K) * 16), dtype=np.uint8), np.full((K, mx.pitch(K)), 255, dtype=np.uint8)
    scales[:, :mx.blocks(K)] = 127
    i = np.arange(K)
    codes[i, i // 2] = 2 << 4 * (i % 2)                    # 1.0
    assert np.array_equal(mx.values_of(codes, scales, K), np.eye(K))
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()


def activations(batch, seed, far, deep):
    """Blocks of magnitudes 2^-far .. 2^far; in each the largest in [1, 2) times that, others down to 2^-deep of it; eight-bit significands, both signs, some zeros."""
    g = np.random.default_rng(seed)
    blocks = mx.blocks(K)
    exponent = -g.integers(0, deep + 1, (batch, blocks, 32)).astype(np.float64)
    exponent[:, :, 0] = 0                                  # column 0 of a block holds the largest binade
    x = g.integers(128, 256, exponent.shape) / 128 * np.exp2(exponent) * np.where(g.random(exponent.shape) < 0.5, -1.0, 1.0)
    x[g.random(x.shape) < 0.1] = 0
    x *= np.exp2(g.integers(-far, far + 1, (batch, blocks, 1)))
    x[:, g.random(blocks) < 0.1] = 0
    x = x.reshape(batch, -1)[:, :K]
    t = torch.from_numpy(x).bfloat16()
    assert np.array_equal(t.double().numpy(), x)
    return t.cuda()


def products(P, ctx, unit, x):
    yield P.llvq_mx_gemm_small_batch(ctx, *unit, K, K, x)
    yield P.llvq_mx_gemv(ctx, *unit, K, K, x[-1].contiguous())[None]


@pytest.mark.parametrize("far", [0, 5, 12, 30, 90])
@pytest.mark.parametrize("batch", BATCHES)
def test_exact_down_to_2_to_the_minus_19_of_the_block(P, ctx, unit, batch, far):
    # binades 0 to 18 below the largest one: every number is above 2^-19 of the largest
    x = activations(batch, batch + far, far, 18)
    for y in products(P, ctx, unit, x):
        assert torch.equal(y.double(), x[-len(y):].double())


@pytest.mark.parametrize("far", [0, 5, 12, 20, 30])
@pytest.mark.parametrize("batch", BATCHES)
def test_off_by_2_to_the_minus_27_of_the_block_below(P, ctx, unit, batch, far):
    x = activations(batch, batch + far, far, 45)
    wide = torch.nn.functional.pad(x.double(), (0, mx.blocks(K) * 32 - K)).view(batch, -1, 32)
    bound = (wide.abs().amax(2, keepdim=True) * 2.0 ** -27).expand(wide.shape).reshape(batch, -1)[:, :K]
    for y in products(P, ctx, unit, x):
        want, off = x[-len(y):].double(), bound[-len(y):]
        half_step = torch.finfo(y.dtype).eps / 2           # the result's rounding; nothing else: the other terms are zeros
        assert ((y.double() - want).abs() <= off + half_step * (want.abs() + off)).all()


@pytest.mark.parametrize("batch", [1, 2, 8, 16])
def test_exact_down_to_2_to_the_minus_31_of_the_chunk(P, ctx, unit, batch):
    # up to 16 rows: numbers of one binade and one 2^31 times as large, in their block or in another; every significand of eight bits
    g = torch.Generator().manual_seed(batch)
    for column in (0, 40, 511, 600):
        x = (torch.randint(128, 256, (batch, K), generator=g) / 128).bfloat16()
        x[:, column] = 2.0 ** 31
        for y in products(P, ctx, unit, x.cuda()):
            assert torch.equal(y.cpu().double(), x[-len(y):].double())


@pytest.mark.parametrize("batch", [1, 3, 16, 20, 40])
@pytest.mark.parametrize("large", [33, 40, 100])
def test_a_channel_that_the_weights_leave_out(P, ctx, batch, large):
    # as a sum: with the large channel's weights zero, what binary32 gives for the others
    n_out, k_in = 70, 1000
    codes, scales = mx.random_matrix(n_out, k_in, seed=5)
    codes[:, 50] = 0                                       # columns 100 and 101
    x = torch.randn((batch, k_in), generator=torch.Generator().manual_seed(batch))
    x[:, 96:128] = 0
    x = torch.where(x.abs() < 2.0 ** -12, 0.0, x)
    x[:, 100] = 2.0 ** large
    x = x.bfloat16()
    w = mx.values_of(codes, scales, k_in)
    y = P.llvq_mx_gemm_small_batch(ctx, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), n_out, k_in, x.cuda()).double().cpu().numpy()
    others = x.double().numpy()
    others[:, 100] = 0
    want, size = others @ w.T, np.abs(others) @ np.abs(w).T
    # 32 columns are summed with at most two truncations of 2^-23 per step of 16, the blocks' sums with one rounding each; half a step of bf16
    slack = 2 * (12 + k_in / 32) * 2.0 ** -23 * size
    assert (np.abs(y - want) <= slack + 2.0 ** -8 * (np.abs(want) + slack)).all()
