"""The operators of channels-last blocks from their definitions, in 64 bits, in plain numpy / torch on the CPU.

Each function returns the exact result and, where the library may round on the way, how far a 32-bit evaluation of the
same formula may be from it (an elementwise bound, derived beside it)."""
from __future__ import annotations

import numpy as np
import torch

BLOCK = 128
U = 2.0 ** -24                                   # half an ulp of 1 in 32 bits


def act(z, kind):
    if kind == "relu":
        return np.where(z < 0, 0.0, z)
    if kind == "silu":
        with np.errstate(over="ignore"):
            return z / (1.0 + np.exp(-z))
    return z


def group_norm(x, G, gamma=None, beta=None, eps=1e-5, kind="none"):
    """(y, bound) of x [N, S, C] in 64 bits.

    The bound, in units of U: the mean of n values summed by several lanes in chains of up to 64 and then in a tree is off by
    at most ~128 mean|x|; a deviation by that and by its own rounding; var by as much, relatively, as the deviations; the last
    four operations add 4 |z|.  gamma scales all of it, an activation has a slope of at most 1.1 and adds 8 |z|."""
    x = np.asarray(x, dtype=np.float64)
    N, S, C = x.shape
    g = x.reshape(N, S, G, C // G)
    mean = g.mean((1, 3), keepdims=True)
    var = ((g - mean) ** 2).mean((1, 3), keepdims=True)
    inv = 1.0 / np.sqrt(var + eps)
    gam = np.ones(C) if gamma is None else np.asarray(gamma, np.float64)
    bet = np.zeros(C) if beta is None else np.asarray(beta, np.float64)
    unit = ((g - mean) * inv).reshape(N, S, C)
    z = unit * gam + bet
    off = np.broadcast_to(128 * np.abs(g).mean((1, 3), keepdims=True) * inv, g.shape).reshape(N, S, C)
    bound = U * (np.abs(gam) * (off * (1 + np.abs(unit)) + 160 * np.abs(unit)) + 12 * np.abs(z) + 4 * np.abs(bet))
    return act(z, kind), 1.1 * bound


def e4m3(t):
    """The nearest 8-bit float (ties to even) of |t| <= 448, by its definition: 3 bits behind the leading one, steps of 2^-9 at the bottom."""
    t = np.asarray(t, np.float64)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(t), 2.0 ** -6))) - 3)
    return np.rint(t / step) * step


def code_step(t):
    """The distance of the codes around t."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(t), 2.0 ** -6))) - 3)


def quantize(x, rows):
    """(code values float32, scales float32), every operation in 32 bits as the definition has it: the result is one bit pattern."""
    x = np.asarray(x, np.float32)
    M, K = x.shape
    mb, kb = -(-M // rows), -(-K // BLOCK)
    scale = np.empty((mb, kb), np.float32)
    code = np.empty((M, K), np.float32)
    for i in range(mb):
        for j in range(kb):
            part = x[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK]
            mag = np.abs(part[~np.isnan(part)])
            a = np.maximum(mag.max() if mag.size else np.float32(0), np.float32(2.0 ** -100)).astype(np.float32)
            scale[i, j] = a / np.float32(448)
            with np.errstate(invalid="ignore"):
                t = part * (np.float32(448) / a)
            code[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK] = torch.from_numpy(np.clip(t, -448, 448)).to(torch.float8_e4m3fn).float().numpy()
    return code, scale


def values(code, scale, rows):
    """What codes [M, K] and the scales of rows x 128 blocks stand for, in 64 bits."""
    M, K = code.shape
    return np.asarray(code, np.float64) * np.asarray(scale, np.float64)[np.arange(M) // rows][:, np.arange(K) // BLOCK]


def product(a, b, bias=None, kind="none", blocks=True, cores8=False):
    """(y, bound) of act(a b^T + bias), a and b 64-bit values.

    The bound: n = K products, exact in 32 bits for codes (one rounding each for 16-bit values), added in any order with 24 bits and
    truncation (2 U each), one multiplication by the scales and one addition a block, the bias, the activation (slope 1.1, 8 U |z|).
    cores8: the products are summed by the 8-bit matrix cores, which line the products of a group up with the largest of them and
    keep 13 bits below its leading one: every product of a block may lose 2^-13 of the largest that the block can have."""
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    K = a.shape[1]
    z = (torch.from_numpy(a) @ torch.from_numpy(b).t().contiguous()).numpy()
    mag = (torch.from_numpy(np.abs(a)) @ torch.from_numpy(np.abs(b)).t().contiguous()).numpy()
    n = 2 * min(K, BLOCK) + 3 * (-(-K // BLOCK)) + 4 if blocks else 2 * K + 4
    lost = 0.0
    if cores8:
        for k in range(0, K, BLOCK):
            part = slice(k, min(K, k + BLOCK))
            lost = lost + (part.stop - k) * 2.0 ** -13 * np.abs(a[:, part]).max(1)[:, None] * np.abs(b[:, part]).max(1)[None, :]
    if bias is not None:
        z = z + bias
        mag = mag + np.abs(bias)
    return act(z, kind), 1.1 * (U * (n * mag + 8 * np.abs(z)) + lost)


# half an ulp of a value relative to it, and the smallest half step, of the output types
ROUND = {"f32": (2.0 ** -24, 2.0 ** -150), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -134)}


def excess(y, ref, bound, ytype):
    """How far outside its allowance the worst element of y is (<= 0: all inside), and where."""
    rel, least = ROUND[ytype]
    y = np.asarray(y, np.float64)
    over = np.abs(y - ref) - (bound + rel * (np.abs(ref) + bound) + least)
    over = np.where(np.isnan(y) != np.isnan(ref), np.inf, np.where(np.isnan(ref), -1.0, over))
    worst = int(np.argmax(over)) if over.size else 0
    return (float(over.flat[worst]), np.unravel_index(worst, over.shape), float(y.flat[worst]), float(ref.flat[worst])) if over.size else (0.0, (), 0.0, 0.0)


# -- products of codes with 16-bit results: how far all of them together may be off -----------------------------

CORE_GROUP, CORE_BITS = 8, 13


def core_sums(ca, sa, cb, sb):
    """The products of codes a [M, K] and b [N, K] (values, scales of 1 x 128 and 128 x 128) as the 8-bit matrix cores sum them: groups of
    eight neighbouring products lined up with the largest of the eight, what lies 13 bits below its leading one cut off; all else exact.
    (Measured on single blocks, the cores' error is 0.5 to 0.7 of this model's: 1.4e-5 of the result for 2.0e-5 on normal values, 2.0e-5 for
    3.6e-5 with one value of a block 30 times the others, 3.4e-5 for 6.3e-5 with 100 times.)"""
    M, K = ca.shape
    N = cb.shape[0]
    ca, cb = np.asarray(ca, np.float64), np.asarray(cb, np.float64)
    out = np.zeros((M, N))
    for k in range(0, K, CORE_GROUP):
        p = ca[:, None, k:k + CORE_GROUP] * cb[None, :, k:k + CORE_GROUP]
        step = np.exp2(np.floor(np.log2(np.maximum(np.abs(p).max(2, keepdims=True), 1e-30))) - CORE_BITS)
        out += (np.trunc(p / step) * step).sum(2) * np.asarray(sa, np.float64)[:, k // BLOCK, None] * np.asarray(sb, np.float64)[np.arange(N) // BLOCK, k // BLOCK][None, :]
    return out


def nearest(z, ytype):
    """z rounded to the type, as 64-bit values."""
    return torch.from_numpy(np.asarray(z, np.float64)).to({"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[ytype]).double().numpy()


def aggregate(y, ref, model, ytype):
    """How many times over its allowance y [n values of the type] is as a whole, against the exact ref and the modelled sums: the larger of

      differences   y - nearest(ref) is a whole number of steps of the type, and not 0 where a rounding boundary lies between the two
                    sums, which for an error e happens |e| / step of the time: the mean of its square is at most the mean of step |e|,
                    so rms(step) rms(e).  e: 1.5 of the model's error, and 2^-20 of the result for sums, scales and their product in 32 bits.
      slope         the part of the error that is in proportion to the result: at most rms(e) of it, and six standard deviations
                    of what the rounding of y leaves in it."""
    y, ref = np.asarray(y, np.float64), np.asarray(ref, np.float64)
    size = np.sqrt((ref ** 2).mean())
    e = 1.5 * np.sqrt(((model - ref) ** 2).mean()) + 2.0 ** -20 * size
    rel = ROUND[ytype][0]
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(ref), 2.0 ** -14 if ytype == "f16" else 2.0 ** -126)))) * 2 * rel
    near = nearest(ref, ytype)
    differences = ((y - near) ** 2).mean() / (np.sqrt((step ** 2).mean()) * e + e ** 2)
    rounding = np.sqrt((((near - ref) * ref) ** 2).mean() / ref.size)
    slope = abs(((y - ref) * ref).mean()) / (e * size + 6 * rounding)
    return float(max(differences, slope))
