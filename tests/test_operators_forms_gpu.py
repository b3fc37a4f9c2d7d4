"""Every form of the operators of channels-last blocks on the GPU, by the form that the library itself says it takes: results, in place,
values that are not finite, streams and graphs."""
import numpy as np
import pytest
import torch

import test_operators_gpu as T
from oracle import operators as O
from paper_2112_15445_amd import binding as B

pytestmark = pytest.mark.gpu


def norm_operands(N, S, C, x_type, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(N, S, C, generator=g, device="cuda") * (0.5 + torch.rand(C, generator=g, device="cuda")) + torch.randn(C, generator=g, device="cuda")
    return x.to(T.T[x_type]), 1 + 0.2 * torch.randn(C, generator=g, device="cuda"), 0.2 * torch.randn(C, generator=g, device="cuda")


# -- group norm: every form that there is -----------------------------------------------------------

# N, S, C, G, type of x, to codes, then the form: kind, lanes of a workgroup, vectors of a lane, x past the cache
NORM_FORMS = [
    (2, 49, 2048, 32, "f16", False, "norm lanes", 256, 4, 0), (2, 1100, 256, 32, "f16", False, "norm lanes", 512, 4, 0),
    (2, 1100, 256, 32, "f32", False, "norm lanes", 512, 16, 0), (3, 3000, 256, 32, "f32", False, "norm lanes", 1024, 16, 0),
    (32, 3136, 256, 32, "f16", False, "norm lanes", 1024, 16, 0), (1340, 49, 256, 32, "f32", False, "norm lanes", 256, 4, 1),
    (300, 250, 256, 32, "f32", False, "norm lanes", 512, 4, 1), (70, 1000, 256, 32, "f32", False, "norm lanes", 512, 16, 1),
    (24, 3001, 256, 32, "f32", False, "norm lanes", 1024, 16, 1), (48, 3001, 256, 32, "bf16", False, "norm lanes", 512, 16, 1),
    (2, 49, 256, 32, "f16", True, "norm lanes", 256, 4, 0), (300, 250, 256, 32, "f16", True, "norm lanes", 512, 16, 0),
    (1340, 49, 256, 32, "f32", True, "norm lanes", 512, 4, 0), (70, 1000, 256, 32, "f16", True, "norm lanes", 1024, 16, 0),
    (70, 1000, 256, 32, "bf16", True, "norm lanes", 1024, 16, 0), (100, 500, 256, 32, "f32", True, "norm lanes", 1024, 16, 0),
    (180, 1000, 256, 32, "f16", True, "norm lanes", 1024, 16, 1),
    (2, 4, 844, 1, "f16", False, "norm sample", 256, 4, 0), (2, 1100, 64, 32, "f16", False, "norm sample", 1024, 4, 0),
    (64, 49, 1040, 16, "f32", False, "norm sample", 1024, 8, 0), (6, 427, 1152, 16, "f32", False, "norm sample", 1024, 8, 0),
    (2, 5, 844, 1, "f16", True, "norm sample", 256, 4, 0), (40, 60, 1152, 12, "f16", True, "norm sample", 1024, 4, 0),
    (64, 49, 1040, 16, "bf16", True, "norm sample", 1024, 8, 0),
    (2, 3000, 48, 3, "f16", False, "norm two", 0, 0, 0), (1, 5000, 7, 1, "f32", False, "norm two", 0, 0, 0), (1, 700, 5000, 2, "bf16", False, "norm two", 0, 0, 0),
    (32, 3136, 256, 32, "bf16", True, "norm two", 0, 0, 0), (7, 837, 360, 30, "bf16", True, "norm two", 0, 0, 0), (2, 500, 200, 8, "f32", True, "norm two", 0, 0, 0),
]


@pytest.mark.parametrize("N,S,C,G,x_type,codes,kind,lanes,held,past", NORM_FORMS)
def test_group_norm_in_every_form(N, S, C, G, x_type, codes, kind, lanes, held, past):
    """The first, a middle and the last sample against the definition."""
    x, gamma, beta = norm_operands(N, S, C, x_type, N + S)
    y_type = "e4m3" if codes else x_type
    op = B.GroupNorm(N, S, C, G, act="silu", x_type=x_type, y_type=y_type)
    l = op.launch()
    assert (l["form"], l["lanes"], l["held"], l["past_cache"]) == (kind, lanes, held, past)
    ws, wp, wn = T.workspace(op)
    assert (wn > 0) == (kind == "norm two")
    row, kb = -(-C // 16) * 16 if codes else C, -(-C // 128)
    y, ys = T.Out(N * S, C, y_type, row), T.Out(N * S, kb, "f32")
    op.forward(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.ptr, ys.ptr if codes else 0, wp, wn, T.stream())
    torch.cuda.synchronize()
    at = sorted({0, N // 2, N - 1})
    ref, bound = O.group_norm(T.host(x[at]), G, T.host(gamma), T.host(beta), 1e-5, "silu")
    got = T.host(y.rows().view(N, S, C)[at] if not codes else torch.stack([y.rows()[n * S:(n + 1) * S] for n in at]))
    if codes:
        scale = T.host(torch.stack([ys.rows()[n * S:(n + 1) * S] for n in at])).astype(np.float64)
        for j in range(kb):
            part = slice(j * 128, (j + 1) * 128)
            a = np.maximum(np.abs(ref[..., part]).max(-1), 2.0 ** -100)
            assert np.all(np.abs(scale[..., j] * 448 - a) <= bound[..., part].max(-1) + 4 * O.U * a), j
            t, c = ref[..., part] / scale[..., j:j + 1], got[..., part].astype(np.float64)
            allowed = 0.5 * O.code_step(np.maximum(np.abs(t), np.abs(c))) + bound[..., part] / scale[..., j:j + 1] + 8 * O.U * np.abs(t)
            assert np.all(np.abs(c - t) <= allowed), j
        ys.check_guard()
    else:
        T.assert_close(got, ref, bound, y_type, (N, S, C, G, x_type))
    y.check_guard(pad=-C % 16 if codes else 0)


IN_PLACE = [  # N, S, C, G, elements between the rows, form in f16 / f32
    (2, 49, 256, 32, 0, "norm lanes"), (2, 3136, 64, 8, 0, "norm lanes"), (2, 4, 844, 1, 4, "norm sample"), (3, 40, 1152, 16, 0, "norm sample"),
    (2, 3000, 48, 3, 0, "norm two"), (1, 5000, 7, 1, 2, "norm two"), (1, 700, 5000, 2, 0, "norm two"),
]


@pytest.mark.parametrize("x_type", ["f16", "f32"])
@pytest.mark.parametrize("N,S,C,G,pad,form", IN_PLACE)
def test_group_norm_in_place_in_every_form(N, S, C, G, pad, form, x_type):
    x, gamma, beta = norm_operands(N, S, C, x_type, 5)
    wide = torch.full((N, S, C + pad), 3.0, device="cuda").to(T.T[x_type])
    wide[..., :C] = x
    strides = (S * (C + pad), C + pad)
    op = B.GroupNorm(N, S, C, G, x_type=x_type, act="relu", x_strides=strides, y_strides=strides)
    assert op.launch()["form"] == form
    ws, wp, wn = T.workspace(op)
    assert (wn > 0) == (form == "norm two")
    y, z = torch.full_like(wide, 3.0), wide.clone()
    for src, dst in ((wide, y), (z, z)):
        op.forward(src.data_ptr(), gamma.data_ptr(), beta.data_ptr(), dst.data_ptr(), 0, wp, wn, T.stream())
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    assert bool((y[..., C:] == 3.0).all())
    ref, bound = O.group_norm(T.host(x), G, T.host(gamma), T.host(beta), 1e-5, "relu")
    T.assert_close(T.host(y[..., :C]), ref, bound, x_type, (N, S, C, G))


NOT_FINITE = [  # N, S, C, G, type, to codes, form
    (2, 40, 64, 8, "f32", False, "norm lanes"), (2, 1100, 256, 32, "f16", False, "norm lanes"), (2, 49, 256, 32, "bf16", True, "norm lanes"),
    (2, 9, 1040, 16, "f16", False, "norm sample"), (3, 40, 1152, 16, "f32", False, "norm sample"), (2, 37, 360, 30, "f16", True, "norm sample"),
    (2, 3000, 48, 3, "f16", False, "norm two"), (2, 5000, 14, 2, "f32", False, "norm two"), (2, 837, 360, 30, "bf16", True, "norm two"),
    (2, 200, 2600, 2, "f32", False, "norm two"),
]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("N,S,C,G,x_type,codes,form", NOT_FINITE)
def test_group_norm_keeps_what_is_not_finite_in_its_group_in_every_form(N, S, C, G, x_type, codes, form, bad):
    """Of a group with such a value all of it is NaN and nothing else: its mean or its deviations are."""
    x, gamma, beta = norm_operands(N, S, C, x_type, 6)
    Cg = C // G
    x[0, S // 2, Cg + Cg // 2] = bad                          # sample 0, group 1
    x[N - 1, S - 1, C - 1] = bad                              # the last sample, position and group
    y_type = "e4m3" if codes else x_type
    op = B.GroupNorm(N, S, C, G, x_type=x_type, y_type=y_type, act="relu")
    assert op.launch()["form"] == form
    ws, wp, wn = T.workspace(op)
    y = B.empty_codes(N * S, C) if codes else torch.empty(N, S, C, dtype=x.dtype, device="cuda")
    ys = torch.empty(N * S, -(-C // 128), device="cuda", dtype=torch.float32)
    op.forward(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.data_ptr(), ys.data_ptr() if codes else 0, wp, wn, T.stream())
    torch.cuda.synchronize()
    nan = np.isnan(T.host(y).reshape(N, S, G, Cg))
    want = np.zeros_like(nan)
    want[0, :, 1] = want[N - 1, :, G - 1] = True
    assert np.array_equal(nan, want)
    if codes:
        assert bool(torch.isfinite(ys).all())                 # (a NaN leaves its block's scale to the others)


# -- products: every form, what is not finite -------------------------------------

# one product of each form (16-bit results; the widest tile has no 32-bit ones)
PRODUCTS = {"rows": (40, 520, 1100), "64": (333, 1000, 1100), "64 split": (300, 700, 3000), "128": (4100, 4100, 272), "128 deep": (2000, 1100, 1000), "256": (4090, 4090, 1100)}


def test_the_shapes_of_the_tests_reach_every_form():
    for form, (M, N, K) in PRODUCTS.items():
        for y_type in ("f16", "bf16"):
            assert B.BlockMatmul(M, N, K, y_type=y_type).launch()["form"] == form
    for y_type, most in (("f16", 10), ("bf16", 10), ("f32", 9)):
        seen = {B.BlockMatmul(M, N, K, y_type=y_type).launch()["form"] for M, N, K in T.MATMUL_SHAPES}
        assert seen | ({"256"} if most == 10 else set()) == set(B.FORMS[4:most])


@pytest.mark.parametrize("y_type", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("form", list(PRODUCTS))
def test_products_keep_what_is_not_finite_in_its_row_and_column(form, y_type):
    """A NaN code of either operand and an infinite scale, in a short last slab and in a whole one."""
    if form == "256" and y_type == "f32":
        return
    M, N, K = PRODUCTS[form]
    assert B.BlockMatmul(M, N, K, y_type=y_type).launch()["form"] == form
    rng = np.random.default_rng(2)
    a = torch.randn(M, K, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    b = torch.randn(N, K, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    (qa, sa), (qb, sb) = B.quantize_blocks_torch(a), B.quantize_blocks_torch(b, 128)
    r = [int(v) for v in rng.permutation(M)[:3]] if form != "rows" else [1, 20, 39]
    c = int(rng.integers(N))
    qa.view(torch.uint8)[r[0], 5] = T.NAN_CODE
    qa.view(torch.uint8)[r[1], K - 1] = T.NAN_CODE            # (the short slab)
    qb.view(torch.uint8)[c, K - 2] = T.NAN_CODE
    sa[r[2], 1] = float("inf")
    got = T.host(B.matmul_blocks_torch(qa, sa, qb, sb, dtype=T.T[y_type]))
    bad = np.zeros((M, N), bool)
    bad[r] = True
    bad[:, c] = True
    assert np.all(np.isfinite(got[~bad]))
    assert np.all(np.isnan(got[r[:2]])) and np.all(np.isnan(got[:, c])) and not np.any(np.isfinite(got[r[2]]))


# -- SiLU ------------------------------------------------------------------------------------------

def silu_is_right(z, y, y_type, what):
    """z / (1 + exp(-z)) of 32-bit z, relative to itself, for z of -87 and more.

    f32: the exponential within 2 ulp (2^-22), one addition, one division: 1.5 * 2^-22.  16 bits: their own rounding; the exponential
    through a 32-bit product z log2(e), whose rounding and constant count |z| 2^-24 each, and a reciprocal, both within one ulp: 2^-21 with
    the rest; numbers below the type's normal ones are not compared."""
    z = z.astype(np.float64)
    ref = z / (1 + np.exp(-z))
    if y_type == "f32":
        allowed = 1.5 * 2.0 ** -22 * np.ones_like(z)
    else:
        allowed = O.ROUND[y_type][0] * (1 + 2.0 ** -8) + 2.0 ** -21 + 2 * np.abs(z) * 2.0 ** -24
    normal = np.abs(ref) >= (2.0 ** -14 if y_type == "f16" else 2.0 ** -126)
    off = np.abs(y - ref)[normal] / np.abs(ref)[normal] / allowed[normal]
    assert off.max() <= 1, (what, y_type, z[normal][off.argmax()], off.max())


@pytest.mark.parametrize("y_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("S,C,G,form", [(49, 256, 32, "norm lanes"), (4, 844, 1, "norm sample"), (3000, 48, 3, "norm two")])
def test_silu_of_the_norm_relative_to_itself(S, C, G, form, y_type):
    """gamma = 0 makes z beta exactly."""
    z = torch.linspace(-87, 87, C).cuda()
    x = torch.randn(2, S, C, device="cuda").to(T.T[y_type])
    op = B.GroupNorm(2, S, C, G, x_type=y_type, act="silu")
    assert op.launch()["form"] == form
    y = B.group_norm_torch(x, G, torch.zeros(C, device="cuda"), z, act="silu")
    assert torch.equal(y, y[:1, :1].expand_as(y))
    silu_is_right(T.host(z), T.host(y[0, 0]), y_type, form)


@pytest.mark.parametrize("y_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", list(PRODUCTS))
def test_silu_of_products_relative_to_itself(form, y_type):
    """Rows of zero codes make z the bias exactly."""
    if form == "256" and y_type == "f32":
        return
    M, N, K = PRODUCTS[form]
    (qa, sa), (qb, sb) = B.quantize_blocks_torch(torch.zeros(M, K, device="cuda")), B.quantize_blocks_torch(torch.randn(N, K, device="cuda"), 128)
    z = torch.linspace(-87, 87, N).cuda()
    y = B.matmul_blocks_torch(qa, sa, qb, sb, bias=z, act="silu", dtype=T.T[y_type])
    assert torch.equal(y, y[:1].expand_as(y))
    silu_is_right(T.host(z), T.host(y[0]), y_type, form)
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    a = torch.zeros(M, K, device="cuda", dtype=torch.float16)
    b = torch.randn(1, N, K, device="cuda").half()
    if K % 8 == 0 and y_type in ("f32", "f16"):
        y = B.matmul_grouped_torch(a, b, off, bias=z, act="silu", dtype=T.T[y_type])
        silu_is_right(T.host(z), T.host(y[M - 1]), y_type, form + " by expert")


# -- streams and graphs ------------------------------------------------------------------------------

def calls():
    """One call of each form that the calls of test_operators_gpu leave out, on its own buffers: (name, run, output, an input)."""
    out = []
    for N, S, C, G, y_type, form in ((2, 4, 844, 1, "f16", "norm sample"), (2, 37, 360, 30, "e4m3", "norm sample"), (2, 1100, 256, 32, "f16", "norm lanes"), (2, 837, 360, 30, "e4m3", "norm two")):
        x, g, b = norm_operands(N, S, C, "f16", 7)
        y, ys = B.empty_codes(N * S, C) if y_type == "e4m3" else torch.empty_like(x), torch.empty(N * S, -(-C // 128), dtype=torch.float32, device="cuda")
        op = B.GroupNorm(N, S, C, G, act="silu", x_type="f16", y_type=y_type)
        assert op.launch()["form"] == form
        ws, wp, wn = T.workspace(op)
        out.append((form, lambda st, op=op, k=(x, g, b, y, ys, ws), wp=wp, wn=wn: op.forward(k[0].data_ptr(), k[1].data_ptr(), k[2].data_ptr(), k[3].data_ptr(), k[4].data_ptr(), wp, wn, st), y, x))
    for form, (M, N, K) in PRODUCTS.items():
        a, sa = B.quantize_blocks_torch(torch.randn(M, K, device="cuda"))
        b, sb = B.quantize_blocks_torch(torch.randn(N, K, device="cuda"), 128)
        y = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
        op = B.BlockMatmul(M, N, K, y_type="bf16", a_row=a.stride(0), b_row=b.stride(0))
        assert op.launch()["form"] == form
        out.append((form, lambda st, op=op, k=(a, sa, b, sb, y): op.forward(k[0].data_ptr(), k[1].data_ptr(), k[2].data_ptr(), k[3].data_ptr(), 0, k[4].data_ptr(), 0, 0, st), y, sa))
        E, counts = 3, [M // 3, 0, M - M // 3]
        off = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")
        ag, bg = torch.randn(M, 256, device="cuda").half(), torch.randn(E, N, 256, device="cuda").half()
        yg = torch.empty(M, N, device="cuda", dtype=torch.float16)
        og = B.GroupedMatmul(M, N, 256, E, a_type="f16")
        out.append((og.launch()["form"] + " by expert", lambda st, op=og, k=(ag, off, bg, yg): op.forward(k[0].data_ptr(), 0, 0, k[1].data_ptr(), k[2].data_ptr(), 0, 0, k[3].data_ptr(), 0, 0, st), yg, ag))
    return out


def test_every_form_on_another_stream_and_in_a_graph():
    """As the test of the same name in test_operators_gpu: inputs change on the stream, then between the replays of a captured call."""
    s = torch.cuda.Stream()
    for name, run, y, x in calls():
        print("case", name, tuple(y.shape), flush=True)
        results = []
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for k in range(3):
                x.mul_(2.0 if k == 1 else 1.0)
                y.view(torch.uint8).zero_()
                run(s.cuda_stream)
                results.append(y.clone())
        s.synchronize()
        assert not torch.equal(results[0].view(torch.uint8), torch.zeros_like(results[0]).view(torch.uint8))
        x.mul_(0.5)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run(s.cuda_stream)
        for k in range(3):
            x.mul_(2.0 if k == 1 else 1.0)
            y.view(torch.uint8).zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y.view(torch.uint8), results[k].view(torch.uint8)), (name, k)
            torch.zeros(1000, device="cuda").sum().item()         # other work between the replays


def test_the_default_type_of_torch_changes_nothing():
    x = torch.randn(2, 40, 320, device="cuda", dtype=torch.float16)
    want = (*B.group_norm_torch(x, 8, codes=True), *B.quantize_blocks_torch(x), *B.quantize_blocks_torch(x, 128))
    torch.set_default_dtype(torch.bfloat16)
    try:
        got = (*B.group_norm_torch(x, 8, codes=True), *B.quantize_blocks_torch(x), *B.quantize_blocks_torch(x, 128))
    finally:
        torch.set_default_dtype(torch.float32)
    for g, w in zip(got, want):
        assert g.dtype == w.dtype and torch.equal(g.float(), w.float())
