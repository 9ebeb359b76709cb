"""Outputs that a call makes itself, on a stream other than the current one: their memory is that stream's, and stays taken while the current one reads it."""
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu
N_OUT, K_IN, BATCH = 256, 480, 8


@pytest.fixture(scope="module")
def calls():
    import paper_2603_11021_b200 as P
    ctx = P.Context(2, 2, device=0)
    nblocks = N_OUT * (K_IN // 24)
    idx = torch.zeros(ctx.index_bytes(nblocks), dtype=torch.uint8, device="cuda")
    gain = torch.full((nblocks,), 0.25, dtype=torch.half, device="cuda")
    book = torch.tensor([1.0, 2.0], device="cuda")
    fields = P.llvq_pack_fields(ctx, torch.zeros(nblocks, dtype=torch.long, device="cuda"), torch.ones(nblocks, dtype=torch.uint8, device="cuda"), 1)
    sort, sort_gemm = P.llvq_sort_blocks(ctx, idx, N_OUT, K_IN), P.llvq_sort_blocks_gemm(ctx, idx, N_OUT, K_IN)
    x = torch.randn((BATCH, K_IN), device="cuda").bfloat16()
    x40 = torch.randn((40, K_IN), device="cuda").bfloat16()
    codes, scales = (torch.from_numpy(a).cuda() for a in mx.random_matrix(N_OUT, K_IN, seed=1))
    xc, xs = P.llvq_mx_quantize(ctx, x)
    table, tokens, dy = torch.randn((50, 96), device="cuda"), torch.randint(0, 50, (70,), device="cuda"), torch.randn((70, 96), device="cuda")
    coder = P.Context(2, 13, device=0)                     # the smallest codes have no encoder
    v = torch.randn((500, 24), device="cuda") * 8
    points, zeros = P.llvq_encode_blocks(coder, v, P.LLVQ_EUCLIDEAN)[0], torch.zeros(nblocks, dtype=torch.long, device="cuda")
    yield {
        "mx_quantize": lambda **s: P.llvq_mx_quantize(ctx, x, **s)[0],
        "mx_quantize_scales": lambda **s: P.llvq_mx_quantize(ctx, x, **s)[1],
        "mx_dequant": lambda **s: P.llvq_mx_dequant_matrix(ctx, codes, scales, N_OUT, K_IN, **s),
        "mx_gemv": lambda **s: P.llvq_mx_gemv(ctx, codes, scales, N_OUT, K_IN, x[0], **s),
        "mx_small_8": lambda **s: P.llvq_mx_gemm_small_batch(ctx, codes, scales, N_OUT, K_IN, x, **s),
        "mx_small_40": lambda **s: P.llvq_mx_gemm_small_batch(ctx, codes, scales, N_OUT, K_IN, x40, **s),
        "mx_gemm": lambda **s: P.llvq_mx_gemm(ctx, xc, xs, BATCH, codes, scales, N_OUT, K_IN, **s),
        "embed": lambda **s: P.llvq_embed(ctx, table, tokens, **s),
        "mx_embed": lambda **s: P.llvq_mx_embed(ctx, codes, scales, N_OUT, K_IN, tokens, **s),
        "embed_grad": lambda **s: P.llvq_embed_grad(ctx, dy, tokens, 50, **s),
        "decode": lambda **s: P.llvq_decode_blocks(ctx, idx, nblocks, **s),
        "dequant": lambda **s: P.llvq_dequant_matrix(ctx, idx, gain, N_OUT, K_IN, P.LLVQ_LAYOUT_ROWWISE, **s),
        "dequant_sg": lambda **s: P.llvq_dequant_matrix_sg(ctx, fields, 1, book, None, N_OUT, K_IN, **s),
        "gemv": lambda **s: P.llvq_gemv(ctx, idx, gain, N_OUT, K_IN, x[0], **s),
        "gemv_sg": lambda **s: P.llvq_gemv_sg(ctx, fields, 1, book, None, N_OUT, K_IN, x[0], **s),
        "gemv_sorted": lambda **s: P.llvq_gemv_sorted(ctx, sort, gain, N_OUT, K_IN, x[0], **s),
        "gemm": lambda **s: P.llvq_gemm_small_batch(ctx, idx, gain, N_OUT, K_IN, x, **s),
        "gemm_sg": lambda **s: P.llvq_gemm_small_batch_sg(ctx, fields, 1, book, None, N_OUT, K_IN, x, **s),
        "gemm_sorted": lambda **s: P.llvq_gemm_small_batch_sorted(ctx, sort_gemm, gain, N_OUT, K_IN, x, **s),
        "sort": lambda **s: P.llvq_sort_blocks(ctx, idx, N_OUT, K_IN, **s),
        "sort_gemm": lambda **s: P.llvq_sort_blocks_gemm(ctx, idx, N_OUT, K_IN, **s),
        "rank": lambda **s: P.llvq_rank_blocks(coder, points, **s),
        "encode": lambda **s: P.llvq_encode_blocks(coder, v, P.LLVQ_EUCLIDEAN, **s)[1],
        "pack": lambda **s: P.llvq_pack_fields(ctx, zeros, None, 0, **s),
    }
    torch.cuda.synchronize()
    assert P.llvq_last_error(ctx) == (0, 0) and P.llvq_last_error(coder) == (0, 0)


@pytest.fixture(scope="module")
def same(calls):
    """Whether two answers of a call are the same; a sorted stream has bytes that nothing defines, so its product is compared."""
    import paper_2603_11021_b200 as P
    ctx = P.Context(2, 2, device=0)
    gain, x = torch.full((N_OUT * (K_IN // 24),), 0.25, dtype=torch.half, device="cuda"), torch.ones((BATCH, K_IN), device="cuda").bfloat16()
    view = {"sort": lambda t: P.llvq_gemv_sorted(ctx, t, gain, N_OUT, K_IN, x[0]), "sort_gemm": lambda t: P.llvq_gemm_small_batch_sorted(ctx, t, gain, N_OUT, K_IN, x)}
    return lambda name, a, b: torch.equal(*(view.get(name, lambda t: t)(t) for t in (a, b)))


NAMES = ["mx_quantize", "mx_quantize_scales", "mx_dequant", "mx_gemv", "mx_small_8", "mx_small_40", "mx_gemm", "embed", "mx_embed", "embed_grad", "decode", "dequant",
         "dequant_sg", "gemv", "gemv_sg", "gemv_sorted", "gemm", "gemm_sg", "gemm_sorted", "sort", "sort_gemm", "rank", "encode", "pack"]


def busy(stream=None):
    with torch.cuda.stream(stream or torch.cuda.current_stream()):
        torch.cuda._sleep(40_000_000)                      # some 20 ms


@pytest.mark.parametrize("name", NAMES)
def test_memory_just_freed_on_the_current_stream_is_not_written_by_another(calls, same, name):
    call, side = calls[name], torch.cuda.Stream()
    want = call()
    torch.cuda.synchronize()
    hold = torch.empty_like(want)
    where = hold.data_ptr()
    busy()
    hold.zero_()                                           # pending when the call is made
    del hold
    got = call(stream=side)
    torch.cuda.synchronize()
    assert got.data_ptr() != where and same(name, got, want)


@pytest.mark.parametrize("name", NAMES)
def test_an_output_dropped_while_it_is_written_is_not_handed_to_the_current_stream(calls, name):
    call, side = calls[name], torch.cuda.Stream()
    torch.cuda.synchronize()
    busy(side)
    got = call(stream=side)
    where, like = got.data_ptr(), torch.empty_like(got, device="meta")
    del got
    other = torch.empty_like(like, device="cuda")
    assert other.data_ptr() != where
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_an_output_that_the_current_stream_still_reads_is_not_written_again(calls, same, name):
    call, side = calls[name], torch.cuda.Stream()
    torch.cuda.synchronize()
    got = call(stream=side)
    side.synchronize()
    where = got.data_ptr()
    busy()
    copy = got.clone()                                     # pending when the output is dropped
    del got
    assert call(stream=side).data_ptr() != where
    torch.cuda.synchronize()
    assert same(name, copy, call())


def test_the_default_stream_given_while_another_is_current(calls, same):
    side = torch.cuda.Stream()
    for name in ("mx_gemv", "embed_grad", "gemv", "sort"):
        want = calls[name]()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = calls[name](stream=torch.cuda.default_stream())
        torch.cuda.synchronize()
        assert same(name, got, want)


def test_captured_on_a_stream_that_forks_from_the_current_one(calls, same):
    for name in ("mx_small_40", "mx_quantize", "embed_grad", "gemm", "sort"):
        want, side = calls[name](), torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            side.wait_stream(torch.cuda.current_stream())
            calls[name](stream=side)                       # dropped at once
            got = calls[name](stream=side)
            torch.cuda.current_stream().wait_stream(side)
            copy = got.clone()
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert same(name, got, want) and same(name, copy, want)
