"""Operators on microscaled 4-bit floating point and on embedding tables, as cases that can be timed.

A case names one operator (`op`), its sizes and types:

  mx_quantize   real matrix -> 4-bit codes and scales (blocks of 32 along a row) -> the values that these stand for
  mx_product    Y = X W^T for 1 to 64 rows of bf16 activations, W held in 4 bits
  mx_linear     the same for a prompt: the activations are quantised to 4 bits too, then both operands meet on the tensor cores
  embed         rows of a table by token, times a scale; the table dense (f32, bf16, f16) or held in 4 bits (mx)
  embed_grad    the gradient of the lookup with respect to a dense table

Where `own` is false, `run` computes them with elementary torch operations; where it is true, by the library's entry points.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

BLOCK = 32                                            # elements that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)        # magnitudes of the 4-bit elements, by their low three bits
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_FLOPS = 2 * 4096 * 28672 * 8192                  # no drawn prompt is larger than the largest listed one
MOST_WEIGHTS = 128256 * 4096
MOST_GRAD_BYTES = 128256 * 4096 * 4


def listed():
    return [
        # The activations of eight requests ahead of a product of 4-bit operands: the smallest call.
        dict(name="quantize_8x4096", op="mx_quantize", rows=8, cols=4096, dtype="bf16"),
        # A whole layer of a checkpoint in binary32, with rows that end inside a block.
        dict(name="quantize_11008x4104_f32", op="mx_quantize", rows=11008, cols=4104, dtype="f32"),
        # One token through the square projection of a 7B decoder.
        dict(name="product_4096x4096_b1", op="mx_product", rows=4096, cols=4096, batch=1, y="bf16"),
        # The output head of an 8B decoder, one token, binary32 logits.
        dict(name="product_128256x4096_b1", op="mx_product", rows=128256, cols=4096, batch=1, y="f32"),
        # A few requests at once, columns that are no multiple of the block.
        dict(name="product_4096x11004_b5", op="mx_product", rows=4096, cols=11004, batch=5, y="bf16"),
        # The widest layer of a 70B-class decoder at the largest small batch.
        dict(name="product_28672x8192_b64", op="mx_product", rows=28672, cols=8192, batch=64, y="bf16"),
        # A short prompt of odd length.
        dict(name="linear_4096x4096_t237", op="mx_linear", rows=4096, cols=4096, tokens=237),
        # A long prompt through the widest layer.
        dict(name="linear_28672x8192_t4096", op="mx_linear", rows=28672, cols=8192, tokens=4096),
        # The next tokens of 64 requests from a bf16 table.
        dict(name="embed_32000x4096_n64", op="embed", vocab=32000, dim=4096, tokens=64, table="bf16", scale=1.0),
        # A batch of prompts from the table that the output head shares, held in 4 bits, scaled by the square root of its width.
        dict(name="embed_mx_128256x4096_n16384", op="embed", vocab=128256, dim=4096, tokens=16384, table="mx", scale=64.0),
        # One step of tuning a small model: short sequences, padding among them.
        dict(name="embed_grad_32000x512_n1000", op="embed_grad", vocab=32000, dim=512, tokens=1000, dtype="bf16", grad="bf16", scale=1.0, padding=0.2),
        # One step on 16384 tokens with the vocabulary of an 8B decoder, binary32 gradient.
        dict(name="embed_grad_128256x4096_n16384", op="embed_grad", vocab=128256, dim=4096, tokens=16384, dtype="bf16", grad="f32", scale=64.0, padding=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _width(rng, lo, hi):
    """A number of columns: half of them ragged."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.5 else max(n // 64, 1) * 64


def draw(rng):
    op = rng.choice(["mx_quantize", "mx_product", "mx_product", "mx_linear", "embed", "embed_grad"])
    if op == "mx_quantize":
        return dict(op=op, rows=_log_int(rng, 1, 16384), cols=_width(rng, 64, 14336), dtype=rng.choice(["f32", "bf16", "f16"]))
    if op == "mx_product":
        batch = rng.choice([1, 1, rng.randint(2, 16), rng.randint(1, 64), 64])
        while True:
            rows, cols = _log_int(rng, 256, 128256), _width(rng, 480, 14336)
            if rows * cols <= MOST_WEIGHTS and rows * cols * batch <= 28672 * 8192 * 64:
                return dict(op=op, rows=rows, cols=cols, batch=batch, y=rng.choice(["f32", "bf16"]) if batch == 1 else "bf16")
    if op == "mx_linear":
        while True:
            rows, cols, tokens = _log_int(rng, 256, 28672), _width(rng, 480, 14336), _log_int(rng, 65, 8192)
            if 2 * rows * cols * tokens <= MOST_FLOPS:
                return dict(op=op, rows=rows, cols=cols, tokens=tokens)
    vocab, dim, scale = _log_int(rng, 500, 128256), _width(rng, 64, 8192), rng.choice([1.0, 0.5, 64.0, math.sqrt(1000.0)])
    if op == "embed":
        tokens = min(_log_int(rng, 1, 65536), 16384 * 4096 // dim)
        return dict(op=op, vocab=vocab, dim=dim, tokens=tokens, table=rng.choice(["f32", "bf16", "f16", "mx", "mx"]), scale=scale)
    while vocab * dim * 4 > MOST_GRAD_BYTES:
        vocab //= 2
    tokens = min(_log_int(rng, 1, 65536), 16384 * 4096 // dim)
    dtype = rng.choice(["f32", "bf16", "f16"])
    return dict(op=op, vocab=vocab, dim=dim, tokens=tokens, dtype=dtype, grad=rng.choice(["f32", dtype]), scale=scale, padding=rng.choice([0.0, 0.3]))


# ---- the 4-bit format ---------------------------------------------------------------------------------------------------------

def _blocks(cols):
    return (cols + BLOCK - 1) // BLOCK


def _pitch(cols):
    """Bytes of a row of scales: whole 16-byte groups."""
    return (_blocks(cols) + 15) // 16 * 16


def _quantize(x):
    """(codes, scales) of a real matrix: scale 2^(floor(log2 of the block's largest magnitude) - 2), elements to the nearest, ties to even, at most 6."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.float(), (0, _blocks(cols) * BLOCK - cols)).view(rows, _blocks(cols), BLOCK)
    exponent = ((v.abs().amax(dim=2).view(torch.int32) >> 23) - 2).clamp(0, 254)
    q = v.abs() * _power_of_two(254 - exponent)[:, :, None]
    code = (q > 0.25).byte() + (q >= 0.75) + (q > 1.25) + (q >= 1.75) + (q > 2.5) + (q >= 3.5) + (q > 5.0)
    code += torch.signbit(v) * 8
    code = code.view(rows, -1, 2)
    return code[:, :, 0] | code[:, :, 1] << 4, torch.nn.functional.pad(exponent.to(torch.uint8), (0, _pitch(cols) - _blocks(cols)))


def _power_of_two(exponent):
    """2^(exponent - 127) in binary32, 0 <= exponent <= 254."""
    e = exponent.to(torch.int32)
    return torch.where(e == 0, 1 << 22, e << 23).view(torch.float32)


@functools.lru_cache(maxsize=None)
def _values_of_bytes():
    """The two elements of a byte of codes, [256, 2]."""
    signed = list(GRID) + [-v for v in GRID]
    return torch.tensor([[signed[b & 15], signed[b >> 4]] for b in range(256)], device="cuda")


def _dequantize(codes, scales, cols):
    """The values in binary32, [rows, cols]."""
    rows = codes.shape[0]
    v = _values_of_bytes()[codes.int()].view(rows, _blocks(cols), BLOCK)
    return (v * _power_of_two(scales[:, :_blocks(cols)])[:, :, None]).view(rows, -1)[:, :cols]


# ---- inputs -------------------------------------------------------------------------------------------------------------------

def _weights(rows, cols, g):
    """Codes and scales of Gaussian weights whose rows differ in size."""
    codes = torch.empty((rows, _blocks(cols) * 16), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, _pitch(cols)), dtype=torch.uint8, device="cuda")
    for r in range(0, rows, 8192):
        n = min(8192, rows - r)
        w = torch.randn((n, cols), generator=g, device="cuda") * (0.02 * torch.exp(0.3 * torch.randn((n, 1), generator=g, device="cuda")))
        codes[r:r + n], scales[r:r + n] = _quantize(w)
    return codes, scales


def _activations(rows, cols, g):
    """Gaussian activations with a few channels that are much larger than the others."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    return (x * torch.where(torch.rand(cols, generator=g, device="cuda") < 0.01, 20.0, 1.0)).bfloat16()


def _tokens(case, g):
    """Tokens by rank as a text has them (the k-th most frequent with a frequency of about 1 / k), spread over the vocabulary."""
    u = torch.rand(case["tokens"], generator=g, device="cuda", dtype=torch.float64)
    rank = ((case["vocab"] + 1.0) ** u - 1).long().clamp(0, case["vocab"] - 1)
    step = int(case["vocab"] * 0.618) | 1
    while math.gcd(step, case["vocab"]) != 1:
        step += 2
    return rank * step % case["vocab"]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op == "mx_quantize":
        x = torch.randn((case["rows"], case["cols"]), generator=g, device="cuda")
        x *= torch.exp(1.5 * torch.randn((case["rows"], 1), generator=g, device="cuda"))
        s["x"] = x.to(TYPES[case["dtype"]])
    elif op in ("mx_product", "mx_linear"):
        s["codes"], s["scales"] = _weights(case["rows"], case["cols"], g)
        s["x"] = _activations(case.get("batch") or case["tokens"], case["cols"], g)
    elif op == "embed":
        s["tokens"] = _tokens(case, g)
        if case["table"] == "mx":
            s["codes"], s["scales"] = _weights(case["vocab"], case["dim"], g)
        else:
            s["table"] = (torch.randn((case["vocab"], case["dim"]), generator=g, device="cuda") * 0.02).to(TYPES[case["table"]])
    else:
        s["tokens"] = _tokens(case, g)
        s["padding_idx"] = -1
        if case["padding"]:
            s["padding_idx"] = case["vocab"] - 1
            s["tokens"][torch.rand(case["tokens"], generator=g, device="cuda") < case["padding"]] = case["vocab"] - 1
        s["dy"] = (torch.randn((case["tokens"], case["dim"]), generator=g, device="cuda") * 1e-3).to(TYPES[case["dtype"]])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _context():
    """A program makes its context once."""
    import paper_2603_11021_b200 as P
    return P.Context(2, 13, device=0)


def _run_own(s):
    import paper_2603_11021_b200 as P
    case, ctx = s["case"], _context()
    op = case["op"]
    if op == "mx_quantize":
        codes, scales = P.llvq_mx_quantize(ctx, s["x"])
        return P.llvq_mx_dequant_matrix(ctx, codes, scales, case["rows"], case["cols"])
    if op == "mx_product":
        rows, cols = case["rows"], case["cols"]
        if case["batch"] == 1:
            return P.llvq_mx_gemv(ctx, s["codes"], s["scales"], rows, cols, s["x"], y_dtype=TYPES[case["y"]]).view(1, rows)
        return P.llvq_mx_gemm_small_batch(ctx, s["codes"], s["scales"], rows, cols, s["x"])
    if op == "mx_linear":
        codes, scales = P.llvq_mx_quantize(ctx, s["x"])
        return P.llvq_mx_gemm(ctx, codes, scales, case["tokens"], s["codes"], s["scales"], case["rows"], case["cols"])
    if op == "embed":
        if case["table"] == "mx":
            return P.llvq_mx_embed(ctx, s["codes"], s["scales"], case["vocab"], case["dim"], s["tokens"], scale=case["scale"])
        return P.llvq_embed(ctx, s["table"], s["tokens"], scale=case["scale"])
    return P.llvq_embed_grad(ctx, s["dy"], s["tokens"], case["vocab"], scale=case["scale"], padding_idx=s["padding_idx"], grad_dtype=TYPES[case["grad"]])


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op = case["op"]
    if op == "mx_quantize":
        return _dequantize(*_quantize(s["x"]), case["cols"]).bfloat16()
    if op == "mx_product":
        y = s["x"].float() @ _dequantize(s["codes"], s["scales"], case["cols"]).T
        return y.to(TYPES[case["y"]])
    if op == "mx_linear":
        x = _dequantize(*_quantize(s["x"]), case["cols"])
        return (x @ _dequantize(s["codes"], s["scales"], case["cols"]).T).bfloat16()
    if op == "embed":
        if case["table"] == "mx":
            return (_dequantize(s["codes"][s["tokens"]], s["scales"][s["tokens"]], case["dim"]) * case["scale"]).bfloat16()
        return (s["table"][s["tokens"]].float() * case["scale"]).to(TYPES[case["table"]])
    dy = s["dy"].float() * (s["tokens"] != s["padding_idx"])[:, None]
    grad = torch.zeros((case["vocab"], case["dim"]), device=dy.device).index_add_(0, s["tokens"], dy)
    return (grad * case["scale"]).to(TYPES[case["grad"]])


def work(case):
    """Bytes: each input read once, each output written once (codes: half a byte an element, and a byte of scale per 32).  Operations: those of the products and sums."""
    op = case["op"]
    size = {"f32": 4, "bf16": 2, "f16": 2, "mx": 17 / 32}
    if op == "mx_quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + size["mx"] + 2), "flops": n}
    if op in ("mx_product", "mx_linear"):
        b = case.get("batch") or case["tokens"]
        nbytes = case["rows"] * case["cols"] * size["mx"] + b * (case["cols"] * 2 + case["rows"] * size[case.get("y", "bf16")])
        return {"bytes": nbytes, "flops": 2 * b * case["rows"] * case["cols"]}
    n = case["tokens"] * case["dim"]
    if op == "embed":
        out = size["bf16"] if case["table"] == "mx" else size[case["table"]]
        return {"bytes": n * (size[case["table"]] + out) + case["tokens"] * 8, "flops": n}
    return {"bytes": n * size[case["dtype"]] + case["vocab"] * case["dim"] * size[case["grad"]] + case["tokens"] * 8, "flops": n}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------

def _exact_elements(codes, scales, cols):
    """Element by element: sign, two bits of exponent, one of mantissa, times the block's power of two."""
    nibble = torch.stack([codes.remainder(16), codes.div(16, rounding_mode="floor")], dim=2).flatten(1)[:, :cols].double()
    sign = 1 - 2 * (nibble >= 8).double()
    low = nibble.remainder(8)
    exponent, mantissa = (low / 2).floor(), low.remainder(2)
    magnitude = torch.where(exponent == 0, mantissa / 2, (1 + mantissa / 2) * torch.exp2(exponent - 1).round())
    power = torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, dim=1)[:, :cols]
    return sign * magnitude * power


def _exact_quantized(x):
    """The values that the quantised matrix stands for."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    middles = torch.tensor([(a + b) / 2 for a, b in zip(GRID, GRID[1:])], dtype=torch.float64, device=x.device)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[1], BLOCK):
        v = x[:, c:c + BLOCK].double()
        exponent = torch.frexp(v.abs().amax(dim=1, keepdim=True)).exponent.double() - 1 - 2      # v = m 2^e, 1/2 <= m < 1
        unit = torch.exp2(exponent.clamp(-127, 127))
        q = v.abs() / unit
        below, upto = torch.bucketize(q, middles), torch.bucketize(q, middles, right=True)
        k = torch.where(below % 2 == 0, below, upto)                                           # on a middle: the even one of the two
        out[:, c:c + BLOCK] = torch.copysign(grid[k] * unit, v)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "mx_quantize":
        return _exact_quantized(s["x"])
    if op in ("mx_product", "mx_linear"):
        x = s["x"].double() if op == "mx_product" else _exact_quantized(s["x"])
        y = torch.empty((x.shape[0], case["rows"]), dtype=torch.float64, device=x.device)
        for r in range(0, case["rows"], 4096):
            y[:, r:r + 4096] = x @ _exact_elements(s["codes"][r:r + 4096], s["scales"][r:r + 4096], case["cols"]).T
        return y
    if op == "embed":
        t = s["tokens"]
        rows = _exact_elements(s["codes"][t], s["scales"][t], case["dim"]) if case["table"] == "mx" else s["table"][t].double()
        return rows * case["scale"]
    order = torch.argsort(s["tokens"], stable=True)
    tokens, dy = s["tokens"][order], s["dy"][order].double()
    sums = torch.cat([torch.zeros((1, case["dim"]), dtype=torch.float64, device=dy.device), dy.cumsum(dim=0)])
    ids, counts = torch.unique_consecutive(tokens, return_counts=True)
    ends = counts.cumsum(0)
    grad = torch.zeros((case["vocab"], case["dim"]), dtype=torch.float64, device=dy.device)
    grad[ids] = sums[ends] - sums[ends - counts]
    if s["padding_idx"] >= 0:
        grad[s["padding_idx"]] = 0
    return grad * case["scale"]
