"""Rows of a table by token and the gradient of that, against float64."""
import numpy as np
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    return P.Context(2, 2, device=0)


def f64(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,dim,n", [(1, 1, 1), (5, 7, 3), (10, 8, 40), (33, 63, 17), (100, 1026, 9), (7, 4096, 5), (1000, 100, 1000)])
@pytest.mark.parametrize("scale", [1.0, 31.622776])
def test_lookup(P, ctx, dtype, vocab, dim, n, scale):
    table = torch.randn((vocab, dim), device="cuda").to(dtype)
    tokens = torch.randint(0, vocab, (n,), device="cuda")
    for t in (tokens, tokens.int()):
        out = P.llvq_embed(ctx, table, t, scale)
        assert out.dtype == dtype and tuple(out.shape) == (n, dim)
        # one product in binary32 and one rounding
        assert torch.equal(out, (table[tokens].float() * torch.tensor(scale, device="cuda")).to(dtype))


@pytest.mark.parametrize("shift", [0, 1, 3, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_tables_and_results_off_the_16_byte_boundaries(P, ctx, dtype, shift):
    for vocab, dim in ((6, 37), (9, 64), (3, 5)):
        store = torch.randn(vocab * dim + shift, device="cuda").to(dtype)
        table = store[shift:].view(vocab, dim)
        tokens = torch.arange(vocab - 1, -1, -1, device="cuda")
        for other in (0, 1, 5):
            buf = torch.full((vocab * dim + other + 4,), 2.0, device="cuda", dtype=dtype)
            P.llvq_embed(ctx, table, tokens, d_out=buf[other:other + vocab * dim])
            assert torch.equal(buf[other:other + vocab * dim].view(vocab, dim), table.flip(0))
            assert (buf[:other] == 2).all() and (buf[other + vocab * dim:] == 2).all()


@pytest.mark.parametrize("vocab,dim,n", [(1, 1, 1), (5, 7, 3), (10, 32, 40), (33, 63, 17), (100, 1026, 9), (50, 4104, 30)])
@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_lookup_in_four_bits(P, ctx, vocab, dim, n, scale):
    codes, scales = mx.random_matrix(vocab, dim, seed=dim, lo=90, hi=150)
    tokens = torch.randint(0, vocab, (n,), device="cuda")
    out = P.llvq_mx_embed(ctx, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), vocab, dim, tokens, scale)
    v = torch.from_numpy(mx.values_of(codes, scales, dim)).float().cuda()          # exact
    assert torch.equal(out, (v[tokens] * torch.tensor(scale, device="cuda")).bfloat16())


def test_tokens_outside_the_table_give_zeros_and_are_counted(P, ctx):
    assert P.llvq_last_error(ctx) == (0, 0)
    table = torch.randn((10, 100), device="cuda")
    tokens = torch.tensor([[3, -1], [10, 9], [1 << 40, 0]], device="cuda")
    out = P.llvq_embed(ctx, table, tokens)
    assert tuple(out.shape) == (3, 2, 100)
    assert (out[0, 1] == 0).all() and (out[1, 0] == 0).all() and (out[2, 0] == 0).all() and torch.equal(out[1, 1], table[9]) and torch.equal(out[2, 1], table[0])
    assert P.llvq_last_error(ctx) == (3, 0)
    c, s = P.llvq_mx_quantize(ctx, table)
    out = P.llvq_mx_embed(ctx, c, s, 10, 100, tokens)
    assert (out[0, 1] == 0).all() and torch.equal(out[1, 1], P.llvq_mx_dequant_matrix(ctx, c, s, 10, 100)[9])
    assert P.llvq_last_error(ctx) == (3, 0)
    P.llvq_embed_grad(ctx, torch.ones((6, 100), device="cuda"), tokens.view(-1), 10)      # -1 is no row by default and not counted
    assert P.llvq_last_error(ctx) == (2, 0)


def reference(dy, tokens, vocab, scale, padding):
    grad, size, count = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros(vocab)
    for t, row in zip(tokens, dy):
        if 0 <= t < vocab and t != padding:
            grad[t] += scale * row
            size[t] += abs(scale) * np.abs(row)
            count[t] += 1
    return grad, size, count


def check_grad(got, dy, tokens, vocab, scale, padding=-1, old=None):
    """A sum of c terms in binary32 takes c roundings of 2^-24 of a partial sum, the product with the scale two more (the scale's own
    rounding among them), the old value one; then half a step of the result's type."""
    grad, size, count = reference(f64(dy), tokens.cpu().numpy(), vocab, scale, padding)
    if old is not None:
        grad, size = grad + f64(old), size + np.abs(f64(old))
    slack = (count[:, None] + 4) * 2.0 ** -24 * size * (1 + 2.0 ** -10)
    step = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).smallest_normal * step                             # below the smallest normal number the step is constant
    assert (np.abs(f64(got) - grad) <= slack + step * (np.abs(grad) + slack) + tiny).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("grad_dtype", TYPES)
@pytest.mark.parametrize("vocab,dim,n", [(1, 1, 1), (7, 5, 64), (7, 24, 65), (300, 256, 700), (1000, 261, 129)])
def test_gradient(P, ctx, dtype, grad_dtype, vocab, dim, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    dy = torch.randn((n, dim), generator=g, device="cuda").to(dtype)
    tokens = (torch.rand(n, generator=g, device="cuda") ** 2 * vocab).long().clamp(max=vocab - 1)
    for t in (tokens, tokens.int()):
        got = P.llvq_embed_grad(ctx, dy, t, vocab, scale=0.7, grad_dtype=grad_dtype)
        assert got.dtype == grad_dtype and tuple(got.shape) == (vocab, dim)
        check_grad(got, dy, tokens, vocab, 0.7)


@pytest.mark.parametrize("kind", ["one token", "runs", "all different", "two halves", "padding only"])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 128, 1000, 4097])
def test_gradient_of_tokens_that_come_often(P, ctx, kind, n):
    vocab, dim, padding = 5000, 40, 11
    i = torch.arange(n, device="cuda")
    tokens = {"one token": torch.full((n,), 4999, device="cuda"), "runs": i // 100, "all different": (i * 7) % vocab, "two halves": (i >= n // 2) * 3,
              "padding only": torch.full((n,), padding, device="cuda")}[kind].long()
    dy = torch.randn((n, dim), device="cuda")
    got = P.llvq_embed_grad(ctx, dy, tokens, vocab, padding_idx=padding)
    check_grad(got, dy, tokens, vocab, 1.0, padding)
    assert (got[padding] == 0).all()


@pytest.mark.parametrize("vocab", [511, 512, 262143, 262144, 300000])
def test_gradient_at_the_borders_between_numbers_of_digits(P, ctx, vocab):
    n = 3000
    tokens = torch.randint(0, vocab, (n,), device="cuda")
    tokens[::7] = vocab - 1
    tokens[::11] = 0
    dy = torch.randn((n, 4), device="cuda")
    got = P.llvq_embed_grad(ctx, dy, tokens, vocab)
    check_grad(got, dy, tokens, vocab, 1.0)


@pytest.mark.parametrize("grad_dtype", TYPES)
def test_gradient_is_added_to_what_is_there(P, ctx, grad_dtype):
    old = torch.randn((50, 264), device="cuda").to(grad_dtype)
    dy = torch.randn((300, 264), device="cuda").bfloat16()
    tokens = torch.randint(0, 40, (300,), device="cuda")
    grad = old.clone()
    assert P.llvq_embed_grad(ctx, dy, tokens, 50, scale=3.0, d_grad=grad, accumulate=True) is not None
    check_grad(grad, dy, tokens, 50, 3.0, old=old)
    assert torch.equal(grad[40:], old[40:])


def test_gradient_is_the_same_every_time_and_writes_nothing_else(P, ctx):
    vocab, dim, n = 2000, 300, 20000
    tokens = (torch.rand(n, device="cuda") ** 4 * vocab).long()
    dy = torch.randn((n, dim), device="cuda").bfloat16()
    buf = torch.full((vocab * dim + 16,), 5.0, device="cuda")
    for shift in (0, 1, 3):
        grad = buf[shift:shift + vocab * dim]
        buf.fill_(5.0)
        P.llvq_embed_grad(ctx, dy, tokens, vocab, d_grad=grad)
        assert (buf[:shift] == 5).all() and (buf[shift + vocab * dim:] == 5).all()
        if shift:
            check_grad(grad.view(vocab, dim), dy, tokens, vocab, 1.0)
    a, b = (P.llvq_embed_grad(ctx, dy, tokens, vocab) for _ in range(2))
    assert torch.equal(a, b)


def test_gradient_against_differences(P, ctx):
    # the lookup is linear in the table: <dy, lookup(d)> = <gradient, d>
    vocab, dim = 30, 72
    tokens = torch.randint(0, vocab, (4, 25), device="cuda")
    table, d = torch.randn((vocab, dim), device="cuda"), torch.randn((vocab, dim), device="cuda")
    dy = torch.randn((4, 25, dim), device="cuda")
    grad = P.llvq_embed_grad(ctx, dy, tokens, vocab, scale=2.0)
    change = P.llvq_embed(ctx, table + d, tokens, 2.0).double() - P.llvq_embed(ctx, table, tokens, 2.0).double()
    lhs, rhs = (dy.double() * change).sum(), (grad.double() * d.double()).sum()
    # table + d is rounded to 2^-24 of a number below 16, each gradient to 100 roundings of a sum below 100 * 16: far below 1e-2 in all
    assert abs(float(lhs - rhs)) < 1e-2


def test_no_tokens_and_no_columns(P, ctx):
    none = torch.empty(0, dtype=torch.long, device="cuda")
    assert tuple(P.llvq_embed(ctx, torch.ones((3, 8), device="cuda"), none).shape) == (0, 8)
    assert (P.llvq_embed_grad(ctx, torch.empty((0, 8), device="cuda"), none, 6) == 0).all()
    grad = torch.ones((6, 8), device="cuda")
    P.llvq_embed_grad(ctx, torch.empty((0, 8), device="cuda"), none, 6, d_grad=grad, accumulate=True)
    assert (grad == 1).all()
    assert tuple(P.llvq_embed_grad(ctx, torch.empty((5, 0), device="cuda"), torch.zeros(5, dtype=torch.long, device="cuda"), 6).shape) == (6, 0)


def test_captured_and_on_another_stream(P, ctx):
    vocab, dim, n = 500, 128, 400
    dy, tokens = torch.randn((n, dim), device="cuda"), torch.randint(0, vocab, (n,), device="cuda")
    want = P.llvq_embed_grad(ctx, dy, tokens, vocab)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    grad = torch.empty_like(want)
    P.llvq_embed_grad(ctx, dy, tokens, vocab, d_grad=grad, stream=side)
    other = P.llvq_embed_grad(ctx, dy, tokens, vocab)           # two calls at once
    side.synchronize()
    assert torch.equal(grad, want) and torch.equal(other, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = P.llvq_embed_grad(ctx, dy, tokens, vocab)
        rows = P.llvq_embed(ctx, again, tokens)
    tokens.copy_(tokens.flip(0))
    dy.copy_(dy.flip(0) * 2)
    graph.replay()
    torch.cuda.synchronize()
    check_grad(again, dy, tokens, vocab, 1.0)
    assert torch.equal(rows, again[tokens])


def test_lookup_then_head_then_gradient(P, ctx):
    # a table in 4 bits serves as embedding and as output head; its master copy gets the gradient of the lookup
    vocab, dim = 1000, 480
    master = torch.randn((vocab, dim), device="cuda") * 0.05
    codes, scales = P.llvq_mx_quantize(ctx, master)
    tokens = torch.randint(0, vocab, (24,), device="cuda")
    x = P.llvq_mx_embed(ctx, codes, scales, vocab, dim, tokens, scale=dim ** 0.5)
    logits = P.llvq_mx_gemm_small_batch(ctx, codes, scales, vocab, dim, x)
    w = P.llvq_mx_dequant_matrix(ctx, codes, scales, vocab, dim)
    assert torch.equal(x, (w[tokens].float() * torch.tensor(dim ** 0.5, device="cuda")).bfloat16())
    want = x.double() @ w.double().T
    size = x.double().abs() @ w.double().abs().T
    assert ((logits.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2 * (12 + dim / 256) * 2.0 ** -23 * size * 1.01).all()
    grad = P.llvq_embed_grad(ctx, x, tokens, vocab, scale=dim ** 0.5)
    check_grad(grad, x, tokens, vocab, dim ** 0.5)
    assert P.llvq_last_error(ctx) == (0, 0)


def test_rows_behind_2_to_the_31_elements(P, ctx):
    vocab, dim = 280000, 8192                              # 4.6 GB in bf16, 9.2 GB of gradient
    table = torch.zeros((vocab, dim), dtype=torch.bfloat16, device="cuda")
    far = torch.tensor([vocab - 1, 5, vocab - 1, 270001], device="cuda")
    table[far] = torch.randn((4, dim), device="cuda").bfloat16()
    assert torch.equal(P.llvq_embed(ctx, table, far), table[far])
    dy = torch.randn((4, dim), device="cuda")
    grad = P.llvq_embed_grad(ctx, dy, far, vocab)
    assert torch.equal(grad[5], dy[1]) and torch.equal(grad[270001], dy[3])
    assert ((grad[vocab - 1] - (dy[0] + dy[2])).abs() <= 2.0 ** -23 * (dy[0].abs() + dy[2].abs())).all()
    assert (grad[[0, 4, 6, 270000, 270002, vocab - 2]] == 0).all()
    del grad, table
    codes, scales = P.llvq_mx_quantize(ctx, torch.ones((1, dim), device="cuda"))
    codes = codes.expand(600000, -1).contiguous()          # 2.5 GB of codes
    scales = scales.expand(600000, -1).contiguous()
    scales[599999] += 1
    x = torch.ones(dim, device="cuda").bfloat16()
    y = P.llvq_mx_gemv(ctx, codes, scales, 600000, dim, x)
    assert (y[:-1] == dim).all() and y[-1] == 2 * dim
    y = P.llvq_mx_gemm_small_batch(ctx, codes, scales, 600000, dim, x.expand(40, -1).contiguous())
    assert (y[:, :-1] == dim).all() and (y[:, -1] == 2 * dim).all()
    out = P.llvq_mx_embed(ctx, codes, scales, 600000, dim, torch.tensor([599999, 0], device="cuda"))
    assert (out[0] == 2).all() and (out[1] == 1).all()
