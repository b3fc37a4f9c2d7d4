"""The operators of a channels-last block of a served network, as cases that can be timed: group norm
with its activation, quantisation to 8-bit floats (e4m3) with a scale for each block of 128, the
matrix product of such operands, and products grouped by expert with ragged sizes.

A case is one call.  prepare() makes what a program holds before it: inputs, weights (quantised once),
output buffers, the operator's description and its workspace.  run() is the call: the library's
kernels where `own` is true, else the same formulas in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

_T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
_BLOCK = 128
_E4M3_MAX = 448.0
_AMAX_FLOOR = 2.0 ** -100


def _norm(name, N, S, C, G, x, y, act, pad=0):
    c = dict(kind="norm", N=N, S=S, C=C, G=G, x=x, y=y, act=act, pad=pad)
    return dict(c, name=name) if name else c


def _quant(name, M, K, rows, x, pad=0):
    c = dict(kind="quant", M=M, K=K, rows=rows, x=x, pad=pad)
    return dict(c, name=name) if name else c


def _matmul(name, M, N, K, y, act="none", bias=False):
    c = dict(kind="matmul", M=M, N=N, K=K, y=y, act=act, bias=bias)
    return dict(c, name=name) if name else c


def _grouped(name, tokens, top, E, N, K, x, y, act="none", bias=False, gather=False, skew=1.0):
    """`tokens` tokens, each with `top` of E experts; `skew`: how unequal the experts' shares are (0 = equal)."""
    c = dict(kind="grouped", tokens=tokens, top=top, E=E, N=N, K=K, x=x, y=y, act=act, bias=bias, gather=gather, skew=skew)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one image in the deepest stage of ResNet-50: 7x7 positions, an interactive request, bound by the launch
        _norm("norm f16 7x7x2048 b1", 1, 49, 2048, 32, "f16", "f16", "silu"),
        # ResNet-50 stage 1, the widest activations of the network, a full batch
        _norm("norm f32 56x56x256 b32", 32, 3136, 256, 32, "f32", "f32", "relu"),
        # odd plane, odd batch, groups of 12 channels, a last block of 104 channels; leaves the product's operand
        _norm("norm bf16 27x31x360 b7 e4m3", 7, 837, 360, 30, "bf16", "e4m3", "silu"),
        # activations of ResNet-50 stage 2 (expanded) on their way into a product
        _quant("quant f16 25088x512", 25088, 512, 1, "f16"),
        # a layer's fp32 weights when a model is loaded: blocks of 128 x 128, the last ones cut
        _quant("quant weights f32 2048x1100", 2048, 1100, 128, "f32"),
        # one token (one position) through a square layer: bound by reading the weights once
        _matmul("matmul 1x4096x4096", 1, 4096, 4096, "bf16"),
        # nothing is a round size, fp32 out
        _matmul("matmul 333x1000x1100 f32", 333, 1000, 1100, "f32", "none", True),
        # ResNet-50 stage 3, expand layer as a pointwise product: short sums, many rows
        _matmul("matmul 6272x1024x256", 6272, 1024, 256, "f16", "relu", True),
        # a prompt of 8192 tokens (or a large batch) through a wide layer: bound by the matrix cores
        _matmul("matmul 8192x8192x4096", 8192, 8192, 4096, "bf16"),
        # eight tokens being decoded, two of 16 experts each: few rows an expert, some without any
        _grouped("experts bf16 8x2 E16", 8, 2, 16, 2048, 1024, "bf16", "bf16", "silu"),
        # a prompt of 4096 tokens, two of 32 experts each, unequal shares
        _grouped("experts f16 4096x2 E32", 4096, 2, 32, 2048, 1024, "f16", "f16", "relu", True),
        # the same in 8-bit floats, rows picked from the tokens by an index
        _grouped("experts e4m3 8192x2 E16", 8192, 2, 16, 4096, 2048, "e4m3", "bf16", "none", False, True),
    ]


def draw(rng):
    """One more case of these ranges: sizes over their logarithm, half of them of no round size."""
    def size(lo, hi, unit=1):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, v // unit * unit) if rng.random() < 0.5 else v

    while True:
        kind = rng.choice(["norm", "quant", "matmul", "matmul", "grouped", "grouped"])
        act, bias = rng.choice(["none", "relu", "silu"]), rng.random() < 0.4
        if kind == "norm":
            G = rng.choice([1, 8, 16, 30, 32, 32, 32])
            C = G * size(1, 2048 // G, 4)
            x = rng.choice(["f32", "f16", "bf16"])
            c = _norm(None, size(1, 64), size(1, 3136), C, G, x, rng.choice([x, x, "e4m3"]), act, rng.choice([0, 0, 8, 3]))
        elif kind == "quant":
            c = _quant(None, size(1, 100352, 64), size(16, 8192, 128), rng.choice([1, 1, 128]), rng.choice(["f32", "f16", "bf16"]), rng.choice([0, 0, 8, 3]))
        elif kind == "matmul":
            M = size(1, 16384, 64) if rng.random() < 0.7 else size(1, 64)
            c = _matmul(None, M, size(16, 8192, 128), size(16, 8192, 128), rng.choice(["f32", "f16", "bf16", "bf16"]), act, bias)
        else:
            top = rng.choice([1, 2, 2, 4])
            E = size(max(2, top), 64, 8)
            x = rng.choice(["f16", "bf16", "e4m3", "e4m3"])
            y = rng.choice(["f32", "bf16", "f16"]) if x == "e4m3" else x
            c = _grouped(None, size(1, 8192, 64), top, max(E, top), size(64, 4096, 128), size(64, 4096, 128), x, y, act, bias,
                         rng.random() < 0.5, rng.choice([0.0, 0.5, 1.0, 2.0]))
        w = work(c)
        if w["flops"] <= 2.8e11 and 1e4 <= w["bytes"] <= 2.1e8:
            return c


# ---------------------------------------------------------------------------------------------
# inputs from the seed
# ---------------------------------------------------------------------------------------------

def _blocks(n):
    return -(-n // _BLOCK)


def _spread(scale, dim, n):
    """A scale for each block of 128 along `dim` as one for each of the n places."""
    return scale.repeat_interleave(_BLOCK, dim).narrow(dim, 0, n)


def _amax(t, rows):
    """max |t| over blocks of `rows` x 128 of a matrix (rows = 1 or 128)."""
    M, K = t.shape
    full = t.new_zeros(-(-M // rows) * rows, _blocks(K) * _BLOCK)
    full[:M, :K] = t.abs()
    return full.view(-1, rows, _blocks(K), _BLOCK).amax((1, 3))


def _codes(t, rows):
    """The quantisation of a 32-bit matrix: (e4m3 values, 32-bit scales)."""
    M, K = t.shape
    a = _amax(t, rows).clamp(min=_AMAX_FLOOR)
    up = _spread(_E4M3_MAX / a, 1, K)
    if rows > 1:
        up = _spread(up, 0, M)
    return (t * up).clamp(-_E4M3_MAX, _E4M3_MAX).to(torch.float8_e4m3fn), a / _E4M3_MAX


def _padded(rows, cols, dtype, pad):
    """A matrix whose rows lie `pad` elements further apart than their length: a part of a wider one."""
    return torch.zeros(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _operand(g, rows, K):
    """A matrix in codes with its rows on 16 bytes, and the scales of 1 x 128 blocks: activations."""
    t = torch.randn(rows, K, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    q = _padded(rows, K, torch.float8_e4m3fn, -K % 16)
    q.copy_(_codes(t, 1)[0])
    return q, _codes(t, 1)[1]


def _weights(g, E, N, K):
    """E matrices in codes with their rows on 16 bytes, and the scales of 128 x 128 blocks."""
    q = torch.zeros(E, N, K + -K % 16, dtype=torch.float8_e4m3fn, device="cuda")[:, :, :K]
    s = torch.empty(E, _blocks(N), _blocks(K), device="cuda")
    for e in range(E):
        codes, s[e] = _codes(torch.randn(N, K, generator=g, device="cuda") * 0.05, 128)
        q[e].copy_(codes)
    return q, s


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(c)
    if c["kind"] == "norm":
        N, S, C = c["N"], c["S"], c["C"]
        # activations of a network: channels of unequal mean and spread
        t = torch.randn(N, S, C, generator=g, device="cuda") * (0.5 + torch.rand(C, generator=g, device="cuda")) + 0.5 * torch.randn(C, generator=g, device="cuda")
        s["x"] = torch.zeros(N, S, C + c["pad"], dtype=_T[c["x"]], device="cuda")[:, :, :C]
        s["x"].copy_(t)
        s["gamma"] = 1 + 0.2 * torch.randn(C, generator=g, device="cuda")
        s["beta"] = 0.2 * torch.randn(C, generator=g, device="cuda")
        if c["y"] == "e4m3":
            s["y"] = _padded(N * S, C, _T["e4m3"], -C % 16)
            s["y_scale"] = torch.empty(N * S, _blocks(C), device="cuda")
        else:
            s["y"] = torch.empty(N, S, C, dtype=_T[c["y"]], device="cuda")
    elif c["kind"] == "quant":
        M, K = c["M"], c["K"]
        t = torch.randn(M, K, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(M, 1, generator=g, device="cuda"))
        s["x"] = _padded(M, K, _T[c["x"]], c["pad"])
        s["x"].copy_(t)
        s["q"] = _padded(M, K, _T["e4m3"], -K % 16)
        s["scale"] = torch.empty(-(-M // c["rows"]), _blocks(K), device="cuda")
    elif c["kind"] == "matmul":
        s["a"], s["a_scale"] = _operand(g, c["M"], c["K"])
        b, b_scale = _weights(g, 1, c["N"], c["K"])
        s["b"], s["b_scale"] = b[0], b_scale[0]
        s["bias_"] = 0.2 * torch.randn(c["N"], generator=g, device="cuda") if c["bias"] else None
        s["out"] = torch.empty(c["M"], c["N"], dtype=_T[c["y"]], device="cuda")
    else:
        E, N, K, T = c["E"], c["N"], c["K"], c["tokens"] * c["top"]
        # a router's choice: `top` experts a token by noisy scores around the experts' own popularity
        score = c["skew"] * torch.randn(E, generator=g, device="cuda") + torch.randn(c["tokens"], E, generator=g, device="cuda")
        expert = score.topk(c["top"], 1).indices.reshape(-1)
        order = expert.sort(stable=True).indices
        counts = torch.bincount(expert, minlength=E)
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["counts"] = counts.tolist()
        s["index"] = (order // c["top"]).to(torch.int32) if c["gather"] else None
        have = c["tokens"] if c["gather"] else T
        s["a_scale"] = s["b_scale"] = None
        if c["x"] == "e4m3":
            s["a"], s["a_scale"] = _operand(g, have, K)
            s["b"], s["b_scale"] = _weights(g, E, N, K)
        else:
            s["a"] = _padded(have, K, _T[c["x"]], -K % 8)
            s["a"].copy_(torch.randn(have, K, generator=g, device="cuda"))
            s["b"] = torch.zeros(E, N, K + -K % 8, dtype=_T[c["x"]], device="cuda")[:, :, :K]
            s["b"].copy_(torch.randn(E, N, K, generator=g, device="cuda") * K ** -0.5)
        s["bias_"] = 0.2 * torch.randn(E, N, generator=g, device="cuda") if c["bias"] else None
        s["out"] = torch.empty(T, N, dtype=_T[c["y"]], device="cuda")
    if own:
        s["op"] = _description(s)
    if own and c["kind"] != "quant":
        s["ws"] = torch.empty(max(s["op"].workspace_size(), 16), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------
# the library's operators
# ---------------------------------------------------------------------------------------------

def _description(s):
    """The operator's description that a program keeps beside its weights."""
    from paper_2112_15445_amd import binding as B
    if s["kind"] == "norm":
        return B.GroupNorm(s["N"], s["S"], s["C"], s["G"], eps=1e-5, act=s["act"], x_type=s["x"].dtype, y_type=s["y"].dtype,
                           x_strides=s["x"].stride()[:2], y_strides=(s["S"] * s["y"].stride(-2), s["y"].stride(-2)))
    if s["kind"] == "quant":
        return B.BlockQuantizer(s["M"], s["K"], rows=s["rows"], x_type=s["x"].dtype, x_row=s["x"].stride(0), q_row=s["q"].stride(0))
    if s["kind"] == "matmul":
        return B.BlockMatmul(s["M"], s["N"], s["K"], y_type=s["out"].dtype, act=s["act"], a_row=s["a"].stride(0), b_row=s["b"].stride(0))
    return B.GroupedMatmul(s["out"].shape[0], s["N"], s["K"], s["E"], a_type=s["a"].dtype, y_type=s["out"].dtype, act=s["act"],
                           a_rows=s["a"].shape[0], a_row=s["a"].stride(0), b_row=s["b"].stride(1))


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _run_own(s):
    stream = torch.cuda.current_stream().cuda_stream
    if s["kind"] == "quant":
        s["op"].forward(s["x"].data_ptr(), s["q"].data_ptr(), s["scale"].data_ptr(), stream)
        return s["q"], s["scale"]
    ws, ws_bytes = s["ws"].data_ptr(), s["ws"].numel()
    if s["kind"] == "norm":
        scale = s.get("y_scale")
        s["op"].forward(s["x"].data_ptr(), s["gamma"].data_ptr(), s["beta"].data_ptr(), s["y"].data_ptr(), _ptr(scale), ws, ws_bytes, stream)
        return s["y"] if scale is None else (s["y"], scale)
    if s["kind"] == "matmul":
        s["op"].forward(s["a"].data_ptr(), s["a_scale"].data_ptr(), s["b"].data_ptr(), s["b_scale"].data_ptr(), _ptr(s["bias_"]),
                        s["out"].data_ptr(), ws, ws_bytes, stream)
        return s["out"]
    s["op"].forward(s["a"].data_ptr(), _ptr(s["a_scale"]), _ptr(s["index"]), s["offsets"].data_ptr(), s["b"].data_ptr(), _ptr(s["b_scale"]),
                    _ptr(s["bias_"]), s["out"].data_ptr(), ws, ws_bytes, stream)
    return s["out"]


# ---------------------------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _values(q, scale, rows):
    """The 32-bit values that codes and the scales of their blocks stand for."""
    up = _spread(scale, -1, q.shape[-1])
    if rows > 1:
        up = _spread(up, -2, q.shape[-2])
    return q.float() * up


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "norm":
        N, S, C, G = s["N"], s["S"], s["C"], s["G"]
        x = s["x"].float().reshape(N, S, G, C // G)
        mean = x.sum((1, 3), keepdim=True) / (S * (C // G))
        d = x - mean
        var = (d * d).sum((1, 3), keepdim=True) / (S * (C // G))
        z = (d / torch.sqrt(var + 1e-5)).reshape(N, S, C) * s["gamma"] + s["beta"]
        y = _act(z, s["act"])
        return _codes(y.reshape(N * S, C), 1) if "y_scale" in s else y.to(s["y"].dtype)
    if s["kind"] == "quant":
        return _codes(s["x"].float(), s["rows"])
    if s["kind"] == "matmul":
        z = _values(s["a"], s["a_scale"], 1) @ _values(s["b"], s["b_scale"], 128).t()
        if s["bias_"] is not None:
            z = z + s["bias_"]
        return _act(z, s["act"]).to(s["out"].dtype)
    a = s["a"].float() if s["a_scale"] is None else _values(s["a"], s["a_scale"], 1)
    b = s["b"].float() if s["b_scale"] is None else _values(s["b"], s["b_scale"], 128)
    if s["index"] is not None:
        a = a[s["index"].long()]
    z = torch.cat([x @ w.t() for x, w in zip(a.split(s["counts"]), b)])
    if s["bias_"] is not None:
        z = z + s["bias_"].repeat_interleave((s["offsets"][1:] - s["offsets"][:-1]).long(), 0, output_size=z.shape[0])
    return _act(z, s["act"]).to(s["out"].dtype)


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(c):
    if c["kind"] == "norm":
        n = c["N"] * c["S"] * c["C"]
        scales = 4 * c["N"] * c["S"] * _blocks(c["C"]) if c["y"] == "e4m3" else 0
        return {"bytes": n * (_SIZE[c["x"]] + _SIZE[c["y"]]) + scales + 8 * c["C"], "flops": 10 * n}
    if c["kind"] == "quant":
        return {"bytes": c["M"] * c["K"] * (_SIZE[c["x"]] + 1) + 4 * -(-c["M"] // c["rows"]) * _blocks(c["K"]), "flops": 3 * c["M"] * c["K"]}
    N, K = c["N"], c["K"]
    if c["kind"] == "matmul":
        M = c["M"]
        return {"bytes": M * K + N * K + 4 * (M + _blocks(N)) * _blocks(K) + M * N * _SIZE[c["y"]] + (4 * N if c["bias"] else 0), "flops": 2 * M * N * K}
    T = c["tokens"] * c["top"]
    have, experts = c["tokens"] if c["gather"] else T, min(c["E"], T)
    scales = 4 * (have + experts * _blocks(N)) * _blocks(K) if c["x"] == "e4m3" else 0
    return {"bytes": (have + experts * N) * K * _SIZE[c["x"]] + scales + T * N * _SIZE[c["y"]] + (4 * T if c["gather"] else 0) + (4 * experts * N if c["bias"] else 0),
            "flops": 2 * T * N * K}


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------

def _exact_act(z, act):
    return z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z


def _exact_quantise(y, rows):
    """Codes (as their values) and scales: the largest magnitude of a block becomes 448; a code keeps 3 bits
    behind the leading one, down to steps of 2^-9, ties to the even neighbour."""
    M, K = y.shape
    bm, bk = torch.arange(M, device="cuda") // rows, torch.arange(K, device="cuda") // _BLOCK
    a = torch.zeros(int(bm[-1]) + 1, K, dtype=torch.float64, device="cuda").index_reduce_(0, bm, y.abs(), "amax")
    a = torch.zeros(a.shape[0], int(bk[-1]) + 1, dtype=torch.float64, device="cuda").index_reduce_(1, bk, a, "amax").clamp(min=_AMAX_FLOOR)
    t = y * (448.0 / a[bm][:, bk])
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(t / step) * step, a / 448.0


def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["kind"] == "norm":
        x = s["x"].double().unflatten(2, (c["G"], -1))
        var, mean = torch.var_mean(x, (1, 3), correction=0, keepdim=True)
        y = _exact_act(((x - mean) * (var + 1e-5).rsqrt()).flatten(2) * s["gamma"].double() + s["beta"].double(), c["act"])
        return _exact_quantise(y.flatten(0, 1), 1) if c["y"] == "e4m3" else y
    if c["kind"] == "quant":
        return _exact_quantise(s["x"].double(), c["rows"])

    def values(q, scale, rows):
        q = q.double()
        if scale is None:
            return q
        m, k = torch.arange(q.shape[0], device="cuda") // rows, torch.arange(q.shape[1], device="cuda") // _BLOCK
        return q * scale.double()[m][:, k]

    bias = None if s["bias_"] is None else s["bias_"].double()
    if c["kind"] == "matmul":
        z = values(s["a"], s["a_scale"], 1) @ values(s["b"], s["b_scale"], 128).t().contiguous()
        return _exact_act(z if bias is None else z + bias, c["act"])
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for e, n in enumerate(s["counts"]):
        pick = s["index"][row:row + n].long() if c["gather"] else torch.arange(row, row + n, device="cuda")
        a = values(s["a"].double()[pick], None if s["a_scale"] is None else s["a_scale"][pick], 1)
        z = a @ values(s["b"][e], None if s["b_scale"] is None else s["b_scale"][e], 128).t().contiguous()
        out[row:row + n] = _exact_act(z if bias is None else z + bias[e], c["act"])
        row += n
    return out
