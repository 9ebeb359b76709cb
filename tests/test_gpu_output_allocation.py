"""Outputs that a call makes itself, as PyTorch's own tools see them: dispatch modes, the profiler, filled memory in deterministic programs."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import mx_util as mx

pytestmark = pytest.mark.gpu


class Allocations(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.shapes = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func is torch.ops.aten.empty.memory_format:
            self.shapes.append((tuple(out.shape), out.dtype))
        return out


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


@pytest.fixture(scope="module")
def ctx(P):
    return P.Context(2, 2, device=0)


@pytest.fixture
def matrix():
    return [torch.from_numpy(a).cuda() for a in mx.random_matrix(8, 40, seed=1)]


@pytest.mark.parametrize("side", [False, True])
def test_a_dispatch_mode_sees_every_output(P, ctx, matrix, side):
    s = {"stream": torch.cuda.Stream()} if side else {}
    x, tokens = torch.zeros((3, 40), device="cuda").bfloat16(), torch.zeros(5, dtype=torch.long, device="cuda")
    idx, gain = torch.zeros(ctx.index_bytes(16), dtype=torch.uint8, device="cuda"), torch.ones(16, dtype=torch.half, device="cuda")
    torch.cuda.synchronize()
    with Allocations() as seen:
        P.llvq_mx_gemv(ctx, *matrix, 8, 40, x[0], **s)
        P.llvq_mx_gemm_small_batch(ctx, *matrix, 8, 40, x, **s)
        P.llvq_mx_embed(ctx, *matrix, 8, 40, tokens, **s)
        P.llvq_embed_grad(ctx, torch.ones((5, 40), device="cuda"), tokens, 8, **s)
        P.llvq_gemv(ctx, idx, gain, 8, 48, torch.zeros(48, device="cuda").bfloat16(), **s)
        P.llvq_decode_blocks(ctx, idx, 16, **s)
    torch.cuda.synchronize()
    for want in (((8,), torch.float32), ((3, 8), torch.bfloat16), ((5, 40), torch.bfloat16), ((8, 40), torch.float32), ((16, 24), torch.int8)):
        assert want in seen.shapes
    assert seen.shapes.count(((8,), torch.float32)) == 2


def test_the_profiler_sees_outputs(P, ctx, matrix):
    x = torch.zeros(40, device="cuda").bfloat16()
    with torch.autograd.profiler.profile() as prof:
        P.llvq_mx_gemv(ctx, *matrix, 8, 40, x)
    torch.cuda.synchronize()
    assert "aten::empty" in [e.name for e in prof.function_events]


def test_memory_that_a_deterministic_program_has_filled(P, ctx, matrix):
    idx, gain = torch.zeros(ctx.index_bytes(16), dtype=torch.uint8, device="cuda"), torch.ones(16, dtype=torch.half, device="cuda")
    before, torch.utils.deterministic.fill_uninitialized_memory = torch.utils.deterministic.fill_uninitialized_memory, True
    torch.use_deterministic_algorithms(True, warn_only=True)
    try:
        w = P.llvq_mx_dequant_matrix(ctx, *matrix, 8, 40, ld=64)
        v = P.llvq_dequant_matrix(ctx, idx, gain, 8, 48, P.LLVQ_LAYOUT_ROWWISE, ld=64)
    finally:
        torch.use_deterministic_algorithms(False)
        torch.utils.deterministic.fill_uninitialized_memory = before
    assert torch.isnan(w[:, 40:]).all() and torch.isfinite(w[:, :40]).all()
    assert torch.isnan(v[:, 48:]).all() and torch.isfinite(v[:, :48]).all()
