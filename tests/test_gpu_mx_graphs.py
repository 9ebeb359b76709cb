"""4-bit products and embedding gradients captured into graphs that are replayed side by side, with inputs that change in between."""
import pytest
import torch

import mx_util as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2603_11021_b200 as P
    return P


def make(P, ctx, kind, seed):
    """(the call, inputs that it reads) of one kind; of two kinds of gradient one orders its tokens by comparison, one by digits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind.startswith("grad"):
        n = int(kind[4:])
        dy, tokens = torch.randn((n, 72), device="cuda", generator=g), (torch.rand(n, device="cuda", generator=g) ** 2 * 3000).long()
        return lambda: P.llvq_embed_grad(ctx, dy, tokens, 3000), dy
    codes, scales = (torch.from_numpy(a).cuda() for a in mx.random_matrix(2000, 1500, seed=seed))
    x = torch.randn((int(kind), 1500), device="cuda", generator=g).bfloat16()
    return lambda: P.llvq_mx_gemm_small_batch(ctx, codes, scales, 2000, 1500, x), x


@pytest.mark.parametrize("kind", ["1", "8", "30", "40", "64", "grad1500", "grad9000"])
def test_two_graphs_at_once(P, kind):
    ctx = P.Context(2, 2, device=0)
    made = [make(P, ctx, kind, seed) for seed in (1, 2)]
    streams, graphs, outs = [torch.cuda.Stream() for _ in made], [], []
    for call, _ in made:
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append([call() for _ in range(5)])
    for factor in (1.0, 2.0):
        for _, x in made:
            x.mul_(factor)
        want = [call() for call, _ in made]
        for o in sum(outs, []):
            o.fill_(-1)
        torch.cuda.synchronize()
        for _ in range(10):
            for s, graph in zip(streams, graphs):
                with torch.cuda.stream(s):
                    graph.replay()
        eager = [call() for call, _ in made]               # and beside calls of their own
        torch.cuda.synchronize()
        for w, os, e in zip(want, outs, eager):
            assert torch.equal(e, w) and all(torch.equal(o, w) for o in os)
    assert P.llvq_last_error(ctx) == (0, 0)
