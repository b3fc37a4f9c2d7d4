"""The operators around a layer of experts without a GPU: structures, refusals, the oracle's own definitions."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import experts as X
from paper_2112_15445_amd import binding as B
from test_operators_host import NULL, P, RANGE, SHAPE, UNSUPPORTED, WORKSPACE, refused

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def refused_back(status, op, *args):
    with pytest.raises(B.SparseConvError) as e:
        op.backward(*args)
    assert e.value.status == status and "backward" in str(e.value), e.value


def test_route_refusals():
    R = B.ExpertRouter
    good, back = [P, P, P, P], [P, P, P, P]
    for status, op in ((SHAPE, R(-1, 8, 2)), (SHAPE, R(1, 0, 1, x_row=1, dx_row=1)), (SHAPE, R(1, 4097, 2)), (SHAPE, R(1, 8, 0)), (SHAPE, R(1, 8, 9)), (SHAPE, R(1, 128, 65)),
                       (SHAPE, R(1, 8, 2, x_row=-1)), (UNSUPPORTED, R(1, 8, 2, x_type="e4m3")), (UNSUPPORTED, R(1, 8, 2, x_type=9)), (UNSUPPORTED, R(1, 8, 2, score=2)),
                       (UNSUPPORTED, R(1, 8, 2, normalize=2)), (UNSUPPORTED, R(1, 8, 2, factor=float("nan"))), (UNSUPPORTED, R(1, 8, 2, factor=float("inf"))),
                       (RANGE, R((1 << 25) + 1, 8, 2))):
        refused(status, op, *good)
        refused_back(status, op, *back)
    refused_back(SHAPE, R(1, 8, 2, dx_row=7), *back)
    for i in (0, 2, 3):
        refused(NULL, R(1, 8, 2), *[0 if j == i else P for j in range(4)])
    for i in range(4):
        refused(UNSUPPORTED, R(1, 8, 2), *[P + 2 if j == i else P for j in range(4)])
        refused_back(NULL, R(1, 8, 2), *[0 if j == i else P for j in range(4)])
        refused_back(UNSUPPORTED, R(1, 8, 2), *[P + 2 if j == i else P for j in range(4)])
    refused(UNSUPPORTED, R(1, 8, 2, x_type="f16"), P + 1, P, P, P)
    R(0, 8, 2).forward(0, 0, 0, 0)
    R(0, 8, 2).backward(0, 0, 0, 0)


def test_sort_refusals():
    S = B.ExpertSort
    good = [P, P, P, P, P, 1 << 30]
    for status, op in ((SHAPE, S(-1, 1, 4)), (SHAPE, S(1, 0, 4)), (SHAPE, S(1, 65, 4)), (SHAPE, S(1, 1, 0)), (SHAPE, S(1, 1, 4097)), (RANGE, S((1 << 24) + 1, 64, 4)),
                       (RANGE, S((1 << 30) + 1, 1, 4)), (RANGE, S(0x7fffffff, 64, 4))):
        refused(status, op, *good)
        with pytest.raises(B.SparseConvError):
            op.workspace_size()
    for i in range(4):
        refused(NULL, S(3, 2, 4), *[0 if j == i else v for j, v in enumerate(good)])
        refused(UNSUPPORTED, S(3, 2, 4), *[v + 2 if j == i else v for j, v in enumerate(good)])
    refused(NULL, S(0, 2, 4), 0, 0, 0, 0)
    big = S(65536, 8, 256)
    need = big.workspace_size()
    assert need and S(1024, 8, 4096).workspace_size() == 0
    refused(WORKSPACE, big, P, P, P, P, 0, 0)
    refused(WORKSPACE, big, P, P, P, P, P, need - 1)
    refused(WORKSPACE, big, P, P, P, P, P + 4, need)
    assert S(1 << 24, 64, 4096).workspace_size() < 1 << 32


def test_gather_refusals():
    R = B.RowGather
    good = [P, P, P]
    for status, op in ((SHAPE, R(-1, 8, 4)), (SHAPE, R(1, 0, 4, y_row=1)), (SHAPE, R(1, 8, -1)), (SHAPE, R(1, 8, 4, x_row=-1)), (SHAPE, R(1, 8, 4, y_row=7)),
                       (UNSUPPORTED, R(1, 8, 4, x_type=4)), (UNSUPPORTED, R(1, 8, 4, x_type=-1)), (RANGE, R((1 << 23) + 1, 8, 4)), (RANGE, R(1, (1 << 28) + 1, 4)),
                       (RANGE, R(1, 8, 4, x_row=1 << 32)), (RANGE, R(1, 8, 4, y_row=1 << 61))):
        refused(status, op, *good)
    for i in range(3):
        refused(NULL, R(1, 8, 4), *[0 if j == i else P for j in range(3)])
        refused(UNSUPPORTED, R(1, 8, 4), *[P + 1 if j == i else P for j in range(3)])
    R(0, 8, 4).forward(0, 0, 0)


def test_combine_refusals():
    R = B.RowCombine
    good, back = [P] * 5, [P] * 6
    for status, op in ((SHAPE, R(-1, 2, 8, 4)), (SHAPE, R(1, 0, 8, 4)), (SHAPE, R(1, 65, 8, 4)), (SHAPE, R(1, 2, 0, 4)), (SHAPE, R(1, 2, 8, -1)), (SHAPE, R(1, 2, 8, 4, x_row=-8)),
                       (SHAPE, R(1, 2, 8, 4, y_row=-1)), (SHAPE, R(1, 2, 8, 4, residual_row=-1)), (UNSUPPORTED, R(1, 2, 8, 4, x_type="e4m3")),
                       (UNSUPPORTED, R(1, 2, 8, 4, x_type="f16", y_type="bf16")), (UNSUPPORTED, R(1, 2, 8, 4, x_type="f32", y_type="f16")), (RANGE, R((1 << 23) + 1, 1, 8, 4)),
                       (RANGE, R(1, 1, (1 << 30) + 1, 4))):
        refused(status, op, *good)
        refused_back(status, op, *back)
    refused(SHAPE, R(1, 2, 8, 4, y_row=7), *good)
    refused_back(SHAPE, R(1, 2, 8, 4, dx_row=7), *back)
    for i in (0, 1, 4):
        refused(NULL, R(1, 2, 8, 4), *[0 if j == i else P for j in range(5)])
    for i in (0, 1, 2):
        refused_back(NULL, R(1, 2, 8, 4), *[0 if j == i else P for j in range(6)])
    for i in range(5):
        refused(UNSUPPORTED, R(1, 2, 8, 4), *[P + 1 if j == i else P for j in range(5)])
    for i in range(6):
        refused_back(UNSUPPORTED, R(1, 2, 8, 4), *[P + 1 if j == i else P for j in range(6)])
    R(0, 2, 8, 4).forward(0, 0, 0, 0, 0)
    R(0, 2, 8, 4).backward(0, 0, 0, 0, 0, 0)
    R(3, 2, 8, 4).backward(P, 0, P, 0, 0, 0)                 # no gradient is wanted


def test_adapters_refusals():
    A = B.Adapters
    good = [P, 0, P, P, P, 0, P, P, P, 1 << 40]
    for status, op in ((SHAPE, A(-1, 16, 32, 8, 2, rows=4)), (SHAPE, A(4, 0, 32, 8, 2, y_row=1)), (SHAPE, A(4, 16, 0, 8, 2, x_row=8, a_row=8)), (SHAPE, A(4, 16, 32, 0, 2, b_row=8)),
                       (SHAPE, A(4, 16, 32, 257, 2)), (SHAPE, A(4, 16, 32, 8, 0)), (SHAPE, A(4, 16, 32, 8, 4097)), (SHAPE, A(4, 16, 32, 8, 2, rows=-1)), (SHAPE, A(4, 16, 32, 8, 2, x_row=24)),
                       (SHAPE, A(4, 16, 32, 8, 2, a_row=24)), (SHAPE, A(4, 16, 32, 16, 2, b_row=8)), (SHAPE, A(4, 16, 32, 8, 2, base_row=-1)), (SHAPE, A(4, 16, 32, 8, 2, y_row=15)),
                       (SHAPE, A(4, 16, 32, 8, 2, a_adapter=8 * 32 - 8)), (SHAPE, A(4, 16, 32, 8, 2, b_adapter=16 * 8 - 8)), (SHAPE, A(4, 16, 32, 8, 2, rows=3)),
                       (UNSUPPORTED, A(4, 16, 32, 8, 2, x_type="f32")), (UNSUPPORTED, A(4, 16, 32, 8, 2, x_type="e4m3")), (UNSUPPORTED, A(4, 16, 32, 8, 2, x_type="f16", y_type="bf16")),
                       (UNSUPPORTED, A(4, 16, 32, 8, 2, x_row=36)), (UNSUPPORTED, A(4, 16, 32, 8, 2, a_row=36)), (UNSUPPORTED, A(4, 16, 32, 8, 2, b_row=12)),
                       (UNSUPPORTED, A(4, 16, 32, 8, 2, a_adapter=8 * 32 + 4)), (UNSUPPORTED, A(4, 16, 32, 8, 2, b_adapter=16 * 8 + 4)), (RANGE, A(4, 16, 1 << 21, 8, 2)),
                       (RANGE, A((1 << 30) + 1, 16, 32, 8, 2)), (RANGE, A(4, 16, 32, 8, 2, b_adapter=1 << 60)), (RANGE, A(1 << 30, 1 << 20, 32, 8, 2))):
        refused(status, op, *good)
    op = A(4, 16, 32, 8, 2)
    for i in (0, 2, 3, 4, 6, 7):
        refused(NULL, op, *[0 if j == i else v for j, v in enumerate(good)])
    for i, by in ((0, 8), (1, 2), (2, 2), (3, 8), (4, 4), (5, 2), (6, 1), (7, 1)):
        refused(UNSUPPORTED, op, *[(v or P) + by if j == i else v for j, v in enumerate(good)])
    need = op.workspace_size()
    for ws in ((0, need), (P, need - 1), (P + 8, need)):
        refused(WORKSPACE, op, *good[:8], *ws)
    A(0, 16, 32, 8, 2).forward(0, 0, 0, 0, 0, 0, 0, 0)       # no rows
    A(5, 16, 32, 8, 2, rows=0).forward(0, P, 0, 0, 0, 0, 0, 0)
    A(0, 16, 32, 8, 2, rows=3).forward(0, 0, 0, 0, 0, 0, P, P)       # no group, and y is base
    refused(NULL, A(0, 16, 32, 8, 2, rows=3), 0, 0, 0, 0, 0, 0, 0, P)
    assert A(0, 16, 32, 8, 2).workspace_size() == 0


STRUCTURES = ["sc_route_experts_t", "sc_sort_by_expert_t", "sc_gather_rows_t", "sc_combine_rows_t", "sc_adapters_t"]


def test_structures_match_the_header(tmp_path):
    lines = "".join('printf("%%zu\\n", sizeof(%s));' % n + "".join('printf("%%zu\\n", offsetof(%s, %s));' % (n, f) for f, _ in getattr(B, n)._fields_) for n in STRUCTURES)
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sparse_conv.h"\nint main(void) {' + lines + "return 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    c = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    assert c == [v for n in STRUCTURES for v in [ctypes.sizeof(getattr(B, n))] + [getattr(getattr(B, n), f).offset for f, _ in getattr(B, n)._fields_]]


def test_names_of_the_forms_match_the_header(tmp_path):
    src = tmp_path / "forms.c"
    src.write_text('#include <stdio.h>\n#include "sparse_conv.h"\nint main(void) { printf("%d %d %d %d\\n", SC_FORM_SORT_ONE, SC_FORM_SORT_CHUNKS, SC_FORM_ADAPTERS_FEW, SC_FORM_ADAPTERS_MANY); return 0; }\n')
    exe = tmp_path / "forms"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(v) for v in subprocess.check_output([str(exe)]).split()] == list(range(len(B.FORMS), len(B.FORMS) + len(B.EXPERT_FORMS)))
    assert B.ExpertSort(8, 2, 16).launch()["form"] == "sort one" and B.ExpertSort(65536, 8, 256).launch()["form"] == "sort chunks"
    assert B.ExpertSort(0, 2, 16).launch()["form"] == "nothing" and B.Adapters(0, 16, 32, 8, 2, rows=4).launch()["form"] == "nothing"
    assert B.Adapters(16, 4096, 4096, 16, 8).launch()["form"] == "adapters few" and B.Adapters(8192, 4096, 4096, 64, 7).launch()["form"] == "adapters many"
    for op in (B.ExpertSort(-1, 1, 4), B.Adapters(4, 16, 32, 257, 2)):
        with pytest.raises(B.SparseConvError):
            op.launch()


def test_expert_kernels_spill_at_most_four_registers():
    """No scratch memory but in the adapters' second launch for few rows, 32-bit results and ranks of 65 to 128: four registers of it (f16), two (bf16).  Without
    that cap of 256 registers, one wave a SIMD, they take 32.7 us for 28.7 (768 rows of rank 128)."""
    import re

    import test_kernel_resources as R
    with open(B.LIB_PATH, "rb") as f:
        data = f.read()
    count = {}
    for name, k in {k[".name"]: k for elf in R._code_objects(data) for k in R._kernels(elf)}.items():
        m = re.search(r"(route_pick|route_gradient|sort_count|sort_scan|sort_place|sort_nothing|gather_rows|combine_rows|combine_gradient|adapters_down|adapters_up|adapters_down_wide|adapters_up_wide)_kernel(I|E)", name)
        if not m:
            continue
        kind = m.group(1)
        count[kind] = count.get(kind, 0) + 1
        capped = re.search(r"adapters_up_kernelILi[12]ELi0ELi4E", name)
        assert k[".vgpr_spill_count"] <= (4 if capped else 0) and k[".private_segment_fixed_size"] <= (20 if capped else 0), name
    # router: 3 types, 5 sizes, with a bias or without (gradient: of whole rows or not); sort: two numbers of experts, one workgroup or chunks; rows: through the caches or
    # past them, back 5 pairs of types (gradients: 3 lengths, 3 choices of what is taken, that of the weights alone stores no rows); adapters: 4 pairs; first launch 3 ranks or, many rows, 10 forms; second 4 ranks
    assert count == {"route_pick": 30, "route_gradient": 30, "sort_count": 1, "sort_scan": 1, "sort_place": 4, "sort_nothing": 1, "gather_rows": 2, "combine_rows": 5 * 2, "combine_gradient": 5 * 3 * 5,
                     "adapters_down": 2 * 3, "adapters_down_wide": 4 * 10, "adapters_up": 4 * 4, "adapters_up_wide": 4 * 4}


# -- the oracle's own definitions ------------------------------------------------------------------

@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalize", [False, True])
def test_oracle_router_against_torch(score, normalize):
    x = torch.randn(20, 9, dtype=torch.float64, generator=torch.Generator().manual_seed(1), requires_grad=True)
    s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
    w, at = s.topk(3, 1)
    w = 2.5 * (w / w.sum(1, keepdim=True) if normalize else w)
    ids, ours, _ = X.route(x.detach().numpy(), 3, score, normalize, 2.5)
    assert np.array_equal(ids, at.numpy()) and np.allclose(ours, w.detach().numpy(), rtol=1e-12)
    dw = torch.randn(20, 3, dtype=torch.float64, generator=torch.Generator().manual_seed(2))
    (w * dw).sum().backward()
    assert np.allclose(X.route_backward(x.detach().numpy(), ids, dw.numpy(), score, normalize, 2.5)[0], x.grad.numpy(), rtol=1e-10, atol=1e-13)


def test_oracle_router_of_what_is_out():
    x = np.array([[1.0, -np.inf, np.nan, 1.0], [-np.inf] * 4, [np.nan] * 4, [-0.0, 0.0, -1.0, -np.inf]])
    ids, w, _ = X.route(x, 3)
    assert ids.tolist() == [[0, 3, -1], [-1] * 3, [-1] * 3, [0, 1, 2]]
    assert w[0].tolist() == [0.5, 0.5, 0.0] and not w[1:3].any()
    ids, w, _ = X.route(x, 2, "sigmoid", True, bias=[0.0, 5.0, 5.0, np.nan])
    assert ids.tolist() == [[0, -1], [-1, -1], [-1, -1], [1, 2]]


def test_oracle_sort_by_its_definition():
    rng = np.random.default_rng(0)
    ids = rng.integers(-2, 7, size=(40, 3))
    offsets, index, position = X.sort(ids, 5)
    assert offsets[0] == 0 and offsets[5] == ((ids >= 0) & (ids < 5)).sum() and not (index[offsets[5]:] + 1).any()
    last = [-1] * 5
    for t in range(40):
        for j in range(3):
            p = position[t, j]
            if 0 <= ids[t, j] < 5:
                assert index[p] == t and offsets[ids[t, j]] <= p < offsets[ids[t, j] + 1] and p > last[ids[t, j]]
                last[ids[t, j]] = p
            else:
                assert p == -1


def test_oracle_combine_and_its_gradients_against_torch():
    rng = np.random.default_rng(3)
    position = X.sort(rng.integers(-1, 4, size=(12, 3)), 4)[2]
    x = torch.from_numpy(rng.normal(size=(36, 10))).requires_grad_()
    w = torch.from_numpy(rng.normal(size=(12, 3))).requires_grad_()
    p = torch.from_numpy(position).long()
    y = (torch.where((p >= 0)[:, :, None], x[p.clamp(min=0)], 0) * w[:, :, None]).sum(1)
    assert np.allclose(X.combine(x.detach().numpy(), position, w.detach().numpy())[0], y.detach().numpy())
    dy = torch.from_numpy(rng.normal(size=(12, 10)))
    (y * dy).sum().backward()
    dx, _, dw, _ = X.combine_backward(dy.numpy(), x.detach().numpy(), position, w.detach().numpy())
    assert np.allclose(dx, x.grad.numpy()) and np.allclose(dw, w.grad.numpy())


# -- how many 16-bit numbers carry the adapters' first product ------------------------------------------------

TERMS_KEPT = {("bf16", "bf16"): (2, 2.0 ** -16), ("f16", "f16"): (2, 2.0 ** -22), ("f16", "f32"): (2, 2.0 ** -22), ("bf16", "f32"): (3, 2.0 ** -24)}


def products_of_24_bits(n, R, N, y_type, seed=0):
    """(x [n, 16], a [R, 16], b [N, R], scale, base [n, N], what base + scale (x a^T) b^T is, the same of magnitudes of the first product alone): all of it 16-bit
    numbers, the first product whole numbers of up to 24 bits times a power of two, so exact in 32 bits however it is summed; each column has one rank, a power of two.  With
    16-bit results base takes the leading bits away, so that the last ones are seen."""
    rng = np.random.default_rng(seed)
    x, a, b = np.zeros((n, 16)), np.zeros((R, 16)), np.zeros((N, R))
    x[:, [1, 6, 12]] = rng.integers(0, 256, size=(n, 3)) * rng.choice([-1, 1], size=(n, 1))
    a[:, [1, 6, 12]] = 2.0 ** np.array([15, 7, -1]) * 2.0 ** -(np.arange(R)[:, None] % 3)
    b[np.arange(N), (7 * np.arange(N) + 3) % R] = 2.0 ** (np.arange(N) % 2)
    scale, h = 2.0 ** -12, x @ a.T
    added = scale * (h @ b.T)
    base = np.zeros((n, N)) if y_type == "f32" else -rounded(added, y_type)
    return x, a, b, scale, base, base + added, scale * (np.abs(h).max(1, keepdims=True) @ np.abs(b).sum(1)[None])


def rounded(v, kind):
    return torch.from_numpy(np.asarray(v)).float().to({"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[kind]).double().numpy()


@pytest.mark.parametrize("x_type,y_type", sorted(TERMS_KEPT))
@pytest.mark.parametrize("R", [16, 250])
def test_a_term_less_is_seen(R, x_type, y_type):
    """What the GPU's results are compared with (test_adapters_first_product_keeps_its_bits) holds with all terms of the first product, and not with one less."""
    x, a, b, scale, base, want, size = products_of_24_bits(60, R, 272, y_type)
    for v, kind in ((x, x_type), (a, x_type), (b, x_type), (base, y_type)):
        assert np.array_equal(rounded(v, kind), v)
    h = x @ a.T
    assert np.array_equal(h.astype(np.float32), h)
    up = 2.0 ** (14 - np.frexp(np.abs(h).max(1, keepdims=True))[1]) if x_type == "f16" else 1.0
    terms, off = TERMS_KEPT[x_type, y_type]
    for n in (terms, terms - 1):
        rest, kept = h * up, 0.0
        for _ in range(n):
            kept, rest = kept + rounded(rest, x_type), rest - rounded(rest, x_type)
        got = rounded(base + scale * ((kept / up) @ b.T), y_type)
        step = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[y_type]
        over = (np.abs(got - want) - (off * size + step * (np.abs(want) + off * size))).max()
        assert over <= 0 if n == terms else over > 0
