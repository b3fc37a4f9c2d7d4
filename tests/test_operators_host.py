"""The operators of channels-last blocks without a GPU: structures, refusals, the oracle's own definitions."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2112_15445_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, UNSUPPORTED, RANGE, WORKSPACE = 1, 2, 4, 5, 7
P = 0x10000                          # an address that is never read: every call here is refused (or has no rows)


def test_structures_match_the_header(tmp_path):
    names = ["sc_group_norm_t", "sc_quantize_blocks_t", "sc_matmul_blocks_t", "sc_matmul_grouped_t"]
    lines = "".join('printf("%%zu\\n", sizeof(%s));' % n + "".join('printf("%%zu\\n", offsetof(%s, %s));' % (n, f) for f, _ in getattr(B, n)._fields_) for n in names)
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "sparse_conv.h"\nint main(void) {' + lines + "return 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    c = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    here = [v for n in names for v in [ctypes.sizeof(getattr(B, n))] + [getattr(getattr(B, n), f).offset for f, _ in getattr(B, n)._fields_]]
    assert c == here


def refused(status, op, *args):
    with pytest.raises(B.SparseConvError) as e:
        op.forward(*args)
    assert e.value.status == status, e.value


def test_group_norm_refusals():
    good = (P, P, P, P, 0, P, 1 << 20)
    N = B.GroupNorm
    refused(SHAPE, N(-1, 4, 32, 4), *good)
    refused(SHAPE, N(1, 4, 32, 0), *good)
    refused(SHAPE, N(1, 4, 32, 5), *good)
    refused(SHAPE, N(1, 4, 0, 1), *good)
    refused(SHAPE, N(1, 4, 32, 4, x_strides=(128, -32)), *good)
    refused(SHAPE, N(1, 4, 32, 4, y_strides=(128, 31)), *good)
    refused(SHAPE, N(2, 4, 32, 4, y_strides=(127, 32)), *good)
    refused(UNSUPPORTED, N(1, 4, 32, 4, x_type=B.SC_ELEM_E4M3), *good)
    refused(UNSUPPORTED, N(1, 4, 32, 4, x_type="f16", y_type="f32"), *good)
    refused(UNSUPPORTED, N(1, 4, 32, 4, act=3), *good)
    refused(UNSUPPORTED, N(1, 4, 32, 4, eps=-1.0), *good)
    refused(UNSUPPORTED, N(1, 4, 32, 4, eps=float("nan")), *good)
    refused(RANGE, N(1, 1 << 26, 64, 4), *good)
    refused(RANGE, N(1 << 16, 1 << 16, 1, 1), *good)
    refused(NULL, N(1, 4, 32, 4), 0, P, P, P, 0, P, 1 << 20)
    refused(NULL, N(1, 4, 32, 4), P, P, P, 0, 0, P, 1 << 20)
    refused(UNSUPPORTED, N(1, 4, 32, 4), P + 1, P, P, P, 0, P, 1 << 20)
    refused(UNSUPPORTED, N(1, 4, 32, 4), P, P + 2, P, P, 0, P, 1 << 20)
    e = N(1, 4, 32, 4, y_type="e4m3")
    refused(NULL, e, P, P, P, P, 0, P, 1 << 20)
    refused(UNSUPPORTED, e, P, P, P, P + 8, P, P, 1 << 20)
    refused(UNSUPPORTED, N(1, 4, 32, 4, y_type="e4m3", y_strides=(160, 40)), P, P, P, P, P, P, 1 << 20)
    refused(SHAPE, N(1, 4, 160, 4, y_type="e4m3", scale_row=1), P, P, P, P, P, P, 1 << 20)
    big = N(32, 3136, 256, 32, x_type="f32")
    need = big.workspace_size()
    if need:
        refused(WORKSPACE, big, P, P, P, P, 0, 0, 0)
        refused(WORKSPACE, big, P, P, P, P, 0, P, need - 1)
        refused(WORKSPACE, big, P, P, P, P, 0, P + 4, need)
    N(0, 4, 32, 4).forward(0, 0, 0, 0)                       # nothing to do
    with pytest.raises(B.SparseConvError):
        N(1, 4, 32, 5).workspace_size()


def test_quantize_refusals():
    Q = B.BlockQuantizer
    refused(SHAPE, Q(-1, 16), P, P, P)
    refused(SHAPE, Q(1, 0, q_row=16, scale_row=1), P, P, P)
    refused(SHAPE, Q(1, 17, q_row=16), P, P, P)
    refused(SHAPE, Q(1, 129, scale_row=1), P, P, P)
    refused(SHAPE, Q(1, 16, x_row=-1), P, P, P)
    refused(UNSUPPORTED, Q(1, 16, rows=64), P, P, P)
    refused(UNSUPPORTED, Q(1, 16, x_type=B.SC_ELEM_E4M3), P, P, P)
    refused(UNSUPPORTED, Q(1, 16, x_type=9), P, P, P)
    refused(UNSUPPORTED, Q(1, 16, q_row=24), P, P, P)
    refused(UNSUPPORTED, Q(1, 16), P + 1, P, P)
    refused(UNSUPPORTED, Q(1, 16), P, P + 8, P)
    refused(UNSUPPORTED, Q(1, 16), P, P, P + 2)
    for i in range(3):
        refused(NULL, Q(1, 16), *[0 if j == i else P for j in range(3)])
    Q(0, 16).forward(0, 0, 0)


def test_matmul_refusals():
    M = B.BlockMatmul
    good = [P, P, P, P, 0, P, P, 1 << 30]
    refused(SHAPE, M(-1, 16, 16), *good)
    refused(SHAPE, M(1, 0, 16, y_row=1), *good)
    refused(SHAPE, M(1, 16, 0, a_row=16, b_row=16, a_scale_row=1, b_scale_row=1), *good)
    refused(SHAPE, M(1, 16, 32, a_row=16), *good)
    refused(SHAPE, M(1, 16, 32, b_row=16), *good)
    refused(SHAPE, M(1, 16, 32, y_row=15), *good)
    refused(SHAPE, M(1, 16, 129, a_scale_row=1), *good)
    refused(SHAPE, M(1, 16, 129, b_scale_row=1), *good)
    refused(UNSUPPORTED, M(1, 16, 32, y_type=B.SC_ELEM_E4M3), *good)
    refused(UNSUPPORTED, M(1, 16, 32, act=-1), *good)
    refused(UNSUPPORTED, M(1, 16, 32, a_row=40), *good)
    refused(UNSUPPORTED, M(1, 16, 32, b_row=33), *good)
    refused(RANGE, M(1, 16, 1 << 22), *good)
    refused(RANGE, M((1 << 30) + 1, 16, 16), *good)
    for i in (0, 1, 2, 3, 5):
        refused(NULL, M(1, 16, 32), *[0 if j == i else v for j, v in enumerate(good)])
    for i, by in ((0, 8), (1, 2), (2, 4), (3, 1), (5, 1)):
        refused(UNSUPPORTED, M(1, 16, 32), *[v + by if j == i else v for j, v in enumerate(good)])
    refused(UNSUPPORTED, M(1, 16, 32), P, P, P, P, P + 2, P, P, 1 << 30)
    M(0, 16, 16).forward(0, 0, 0, 0, 0, 0)


def test_grouped_refusals():
    G = B.GroupedMatmul
    good = [P, P, 0, P, P, P, 0, P, P, 1 << 30]
    refused(SHAPE, G(-1, 16, 16, 1), *good)
    refused(SHAPE, G(1, 16, 16, 0), *good)
    refused(SHAPE, G(1, 16, 16, 4097), *good)
    refused(SHAPE, G(1, 16, 32, 2, b_expert=16 * 32 - 8), *good)
    refused(SHAPE, G(4, 16, 32, 2, a_rows=3), *good)                       # without an index
    refused(SHAPE, G(4, 16, 32, 2, a_row=24), *good)
    refused(SHAPE, G(4, 16, 256, 2, a_type="e4m3", a_scale_row=1), *good)
    refused(SHAPE, G(4, 256, 256, 2, a_type="e4m3", b_scale_expert=3), *good)
    refused(UNSUPPORTED, G(4, 16, 32, 2, a_type="f32"), *good)
    refused(UNSUPPORTED, G(4, 16, 32, 2, a_type="f16", y_type="bf16"), *good)
    refused(UNSUPPORTED, G(4, 16, 32, 2, act=7), *good)
    refused(UNSUPPORTED, G(4, 16, 32, 2, a_row=36), *good)
    refused(UNSUPPORTED, G(4, 16, 32, 2, b_expert=16 * 32 + 4), *good)
    refused(RANGE, G(4, 16, 1 << 21, 2), *good)
    for i in (0, 3, 4, 7):
        refused(NULL, G(4, 16, 32, 2), *[0 if j == i else v for j, v in enumerate(good)])
    for i in (1, 5):
        refused(NULL, G(4, 16, 32, 2, a_type="e4m3"), *[0 if j == i else v for j, v in enumerate(good)])
    for i, by in ((0, 8), (3, 2), (4, 4), (7, 1)):
        refused(UNSUPPORTED, G(4, 16, 32, 2), *[v + by if j == i else v for j, v in enumerate(good)])
    G(0, 16, 16, 3).forward(0, 0, 0, 0, 0, 0, 0, 0)


@pytest.mark.parametrize("bad", [b"0123456789abcdef", "text", 1.5, ctypes.c_int64(0)])
def test_operators_take_integers_for_their_pointers(bad):
    for op, n in ((B.GroupNorm(0, 1, 8, 1), 8), (B.BlockQuantizer(0, 16), 4), (B.BlockMatmul(0, 16, 16), 9), (B.GroupedMatmul(0, 16, 16, 1), 11)):
        op.forward(*[0] * n)
        for i in range(n):
            with pytest.raises(TypeError):
                op.forward(*[bad if j == i else 0 for j in range(n)])


def test_names_of_types_and_activations():
    with pytest.raises(KeyError):
        B.GroupNorm(1, 1, 8, 1, x_type="f64")
    with pytest.raises(KeyError):
        B.GroupNorm(1, 1, 8, 1, x_type=torch.float64)
    with pytest.raises(KeyError):
        B.BlockMatmul(1, 16, 16, act="gelu")


# -- the oracle's own definitions ------------------------------------------------------------------

def test_oracle_code_rounding_against_torch():
    t = np.concatenate([np.linspace(-448, 448, 20001), np.linspace(-0.1, 0.1, 20001), [2.0 ** -10, 3 * 2.0 ** -10, 0.0, 17.0, 19.0]]).astype(np.float32)
    assert np.array_equal(O.e4m3(t), torch.from_numpy(t).to(torch.float8_e4m3fn).double().numpy())


def test_oracle_group_norm_against_torch():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(2, 12, 24))
    g, b = rng.normal(size=24), rng.normal(size=24)
    ref = torch.nn.functional.group_norm(torch.from_numpy(x).permute(0, 2, 1), 6, torch.from_numpy(g), torch.from_numpy(b), 1e-3).permute(0, 2, 1).numpy()
    assert np.allclose(O.group_norm(x, 6, g, b, 1e-3)[0], ref, rtol=1e-12, atol=1e-12)
    assert np.allclose(O.group_norm(x, 6, g, b, 1e-3, "silu")[0], torch.nn.functional.silu(torch.from_numpy(ref)).numpy(), rtol=1e-12, atol=1e-12)


def test_oracle_quantisation_is_the_nearest_code():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(130, 200)).astype(np.float32)
    for rows in (1, 128):
        code, scale = O.quantize(x, rows)
        v = O.values(code, scale, rows)
        s = scale.astype(np.float64)[np.arange(130) // rows][:, np.arange(200) // 128]
        assert np.all(np.abs(v - x) <= s * (0.5 * O.code_step(np.abs(x) / s) + 1e-4))
        assert np.abs(code).max() == 448


def test_a_wrong_scale_block_is_seen():
    """The bounds are tight enough for a mistake: the neighbouring block's scale, a dropped last column, a group's bias."""
    rng = np.random.default_rng(2)
    ca, sa = O.quantize(rng.normal(size=(20, 300)).astype(np.float32), 1)
    cb, sb = O.quantize(rng.normal(size=(30, 300)).astype(np.float32), 128)
    ref, bound = O.product(O.values(ca, sa, 1), O.values(cb, sb, 128))
    for wrong in (O.product(O.values(ca, np.roll(sa, 1, 1), 1), O.values(cb, sb, 128))[0],
                  O.product(O.values(ca, sa, 1)[:, :-1], O.values(cb, sb, 128)[:, :-1])[0]):
        assert O.excess(wrong, ref, bound, "f32")[0] > 0 and O.excess(wrong, ref, bound, "bf16")[0] > 0
    assert O.excess(ref, ref, bound, "f32")[0] <= 0


def test_operator_kernels_spill_at_most_two_registers():
    """No scratch memory but in the widest group norm form that leaves codes of two-byte inputs (two registers of it)."""
    import re

    import test_kernel_resources as R
    with open(B.LIB_PATH, "rb") as f:
        data = f.read()
    seen = {}
    for elf in R._code_objects(data):
        for k in R._kernels(elf):
            m = re.search(r"(matmul_tile|matmul_rows|norm_resident|norm_stats|norm_apply|quantize_rows|quantize_tiles)_kernelI", k[".name"])
            if m:
                seen[k[".name"]] = (m.group(1), k)
    count = {}
    for name, (kind, k) in seen.items():
        count[kind] = count.get(kind, 0) + 1
        assert k[".vgpr_spill_count"] <= (2 if kind == "norm_resident" else 0) and k[".private_segment_fixed_size"] <= (16 if kind == "norm_resident" else 0), name
        assert k[".vgpr_count"] + k.get(".agpr_count", 0) <= 256, name
    # types of operands and results: 10 (3 of codes whole, 7 grouped); tiles: 5 each and the widest in 8; group norm: 6 pairs, 3 activations, 4 sizes
    assert count == {"matmul_tile": 10 * 4 + 8, "matmul_rows": 10, "norm_resident": 72, "norm_stats": 3, "norm_apply": 18, "quantize_rows": 3, "quantize_tiles": 3}


def test_whole_sample_norm_kernels_do_not_spill():
    import re

    import test_kernel_resources as R
    with open(B.LIB_PATH, "rb") as f:
        data = f.read()
    seen = {k[".name"]: k for elf in R._code_objects(data) for k in R._kernels(elf) if re.search(r"norm_sample_kernelI", k[".name"])}
    for name, k in seen.items():
        assert k[".vgpr_spill_count"] == 0 and k[".private_segment_fixed_size"] == 0, name
        assert k[".vgpr_count"] + k.get(".agpr_count", 0) <= 128, name
    assert len(seen) == 6 * 3 * 3         # pairs of types, activations, sizes
