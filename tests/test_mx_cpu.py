"""Microscaled 4-bit matrices and embedding tables: what the host settles and refuses, without a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import mx_util as mx


@pytest.fixture(scope="module")
def P():
    from paper_2603_11021_b200 import build
    build.build()
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    return P.Context(2, 2, device=-1)


@pytest.mark.parametrize("cols", [0, 1, 31, 32, 33, 480, 511, 512, 513, 4104, 1 << 31])
def test_pitches(P, cols):
    assert P.llvq_mx_code_pitch(cols) == mx.blocks(cols) * 16
    assert P.llvq_mx_scale_pitch(cols) == mx.pitch(cols)
    assert P.llvq_mx_code_pitch(-1) == 0 and P.llvq_mx_scale_pitch(-1) == 0


def test_workspace_of_the_gradient(P):
    L = P.load_library()
    assert L.llvq_embed_grad_bytes(0, 8) == 0 and L.llvq_embed_grad_bytes(8, 0) == 0 and L.llvq_embed_grad_bytes(1 << 31, 8) == 0
    # lists of keys and positions, twice; two sums per piece of 8 positions at the smallest, 32 at the largest, for columns rounded up to 256
    for n, dim, piece in ((1, 1, 8), (64, 512, 8), (65, 513, 8), (100000, 4096, 32)):
        lists, pieces, padded = 4 * (-(-n * 4 // 256) * 256), -(-n // piece), -(-dim // 256) * 256
        assert L.llvq_embed_grad_bytes(n, dim) == lists + pieces * 2 * padded * 4


def test_the_reference_of_the_tests_quantizes_what_it_should():
    x = np.zeros((1, 40))
    x[0, :8] = [6.0, 7.9, -5.0, 2.5, 0.25, 0.75, -0.2, 3.5]
    codes, scales, v = mx.quantize(x)
    assert scales[0, 0] == 127 and v[0, :8].tolist() == [6.0, 6.0, -4.0, 2.0, 0.0, 1.0, -0.0, 4.0]
    assert np.array_equal(mx.values_of(codes, scales, 40), v)
    assert codes[0, 0] == 7 | 7 << 4 and codes[0, 1] == 14 | 4 << 4


def test_host_only_context_refuses_to_launch(P, ctx):
    L, vp = ctx._lib, ctypes.c_void_p(4096)
    assert L.llvq_device(ctx._h) == -1 and L.llvq_device(None) == -1
    assert L.llvq_mx_quantize(ctx._h, vp, 0, 1, 32, 32, vp, vp, None) == 1
    assert L.llvq_mx_dequant_matrix(ctx._h, vp, vp, 1, 32, vp, 32, None) == 1
    assert L.llvq_mx_gemv(ctx._h, vp, vp, 1, 32, vp, vp, 0, None) == 1
    assert L.llvq_mx_gemm_small_batch(ctx._h, vp, vp, 1, 32, vp, 1, vp, vp, None) == 1
    assert L.llvq_mx_small_batch_bytes(ctx._h, 128, 128, 4) == 0 and L.llvq_mx_small_batch_bytes(None, 128, 128, 4) == 0
    assert L.llvq_mx_gemm(ctx._h, vp, vp, 1, vp, vp, 1, 32, vp, None) == 1
    assert L.llvq_embed(ctx._h, vp, 0, 1, 1, vp, 8, 1, 1.0, vp, None) == 1
    assert L.llvq_mx_embed(ctx._h, vp, vp, 1, 1, vp, 8, 1, 1.0, vp, None) == 1
    assert L.llvq_embed_grad(ctx._h, vp, 0, vp, 8, 1, 1, 1, 1.0, -1, 0, vp, 0, vp, None) == 1


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def test_arguments_are_checked_before_the_device(P, ctx):
    bf, codes, scales = torch.bfloat16, u8(4, 32), u8(4, 16)
    with pytest.raises(AssertionError):
        P.llvq_mx_dequant_matrix(ctx, codes, scales, 4, 65)                 # codes too short
    with pytest.raises(AssertionError):
        P.llvq_mx_dequant_matrix(ctx, u8(4, 17 * 16), scales, 4, 17 * 32)   # scales too short
    with pytest.raises(AssertionError):
        P.llvq_mx_dequant_matrix(ctx, codes.view(torch.int8), scales, 4, 64)
    with pytest.raises(AssertionError):
        P.llvq_mx_dequant_matrix(ctx, codes, scales, 4, 64, ld=63)
    with pytest.raises(AssertionError):
        P.llvq_mx_dequant_matrix(ctx, codes, scales, -1, 64)
    with pytest.raises(AssertionError):
        P.llvq_mx_gemv(ctx, codes, scales, 4, 64, torch.zeros(63, dtype=bf))
    with pytest.raises(AssertionError):
        P.llvq_mx_gemv(ctx, codes, scales, 4, 64, torch.zeros(64))
    with pytest.raises(AssertionError):
        P.llvq_mx_gemv(ctx, codes, scales, 4, 64, torch.zeros(64, dtype=bf), y_dtype=torch.float16)
    with pytest.raises(AssertionError):
        P.llvq_mx_gemm_small_batch(ctx, codes, scales, 4, 64, torch.zeros((2, 63), dtype=bf))
    with pytest.raises(P.LlvqError) as e:
        P.llvq_mx_gemm_small_batch(ctx, codes, scales, 4, 64, torch.zeros((65, 64), dtype=bf))
    assert e.value.status == 3
    for tokens, n_out, k_in, y in ((5, 4, 64, None), (4, 5, 64, None), (4, 4, 65, None), (-1, 4, 64, None), (4, 4, -1, None), (4, 4, 64, torch.zeros(15, dtype=bf)),
                                   (4, 4, 64, torch.zeros(16))):
        with pytest.raises(AssertionError):
            P.llvq_mx_gemm(ctx, codes, scales, tokens, codes, scales, n_out, k_in, y)
    with pytest.raises(AssertionError):
        P.llvq_embed(ctx, torch.zeros((4, 8), dtype=torch.float64), torch.zeros(3, dtype=torch.long))
    with pytest.raises(AssertionError):
        P.llvq_embed(ctx, torch.zeros((4, 8)), torch.zeros(3, dtype=torch.int16))
    with pytest.raises(AssertionError):
        P.llvq_embed(ctx, torch.zeros((4, 8)), torch.zeros(3, dtype=torch.long), d_out=torch.zeros(23))
    with pytest.raises(AssertionError):
        P.llvq_mx_embed(ctx, codes, scales, 5, 64, torch.zeros(3, dtype=torch.long))
    with pytest.raises(AssertionError):
        P.llvq_embed_grad(ctx, torch.zeros((3, 8)), torch.zeros(4, dtype=torch.long), 5)
    with pytest.raises(AssertionError):
        P.llvq_embed_grad(ctx, torch.zeros((3, 8)), torch.zeros(3, dtype=torch.long), 5, grad_dtype=torch.float64)
    with pytest.raises(AssertionError):
        P.llvq_embed_grad(ctx, torch.zeros((3, 8)), torch.zeros(3, dtype=torch.long), 5, accumulate=True)
    with pytest.raises(AssertionError):
        P.llvq_embed_grad(ctx, torch.zeros((3, 8)), torch.zeros(3, dtype=torch.long), 5, d_grad=torch.zeros(39))


def test_host_tensors_are_refused(P, ctx):
    bf, long = torch.bfloat16, torch.long
    for f in (lambda: P.llvq_mx_quantize(ctx, torch.zeros((4, 64))),
              lambda: P.llvq_mx_dequant_matrix(ctx, u8(4, 32), u8(4, 16), 4, 64),
              lambda: P.llvq_mx_gemv(ctx, u8(4, 32), u8(4, 16), 4, 64, torch.zeros(64, dtype=bf)),
              lambda: P.llvq_mx_gemm_small_batch(ctx, u8(4, 32), u8(4, 16), 4, 64, torch.zeros((2, 64), dtype=bf)),
              lambda: P.llvq_mx_gemm(ctx, u8(4, 32), u8(4, 16), 4, u8(4, 32), u8(4, 16), 4, 64),
              lambda: P.llvq_embed(ctx, torch.zeros((4, 8)), torch.zeros(3, dtype=long)),
              lambda: P.llvq_mx_embed(ctx, u8(4, 32), u8(4, 16), 4, 64, torch.zeros(3, dtype=long)),
              lambda: P.llvq_embed_grad(ctx, torch.zeros((3, 8)), torch.zeros(3, dtype=long), 5)):
        with pytest.raises(TypeError, match="contiguous CUDA tensor"):
            f()
