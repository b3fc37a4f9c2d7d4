"""Sizes and distances at the ends of their types: the operators refuse what they could not address.  No call here gets as far as a launch."""
import pytest

from paper_2112_15445_amd import binding as B

SHAPE, UNSUPPORTED, RANGE, WORKSPACE = 2, 4, 5, 7
P = 0x10000                          # an address that is never read


def refused(status, op, *args):
    with pytest.raises(B.SparseConvError) as e:
        op.forward(*args)
    assert e.value.status == status, e.value


@pytest.mark.parametrize("a_type", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("far", [1 << 22, 1 << 31, 1 << 61, 1 << 62])
def test_grouped_distances_are_compared_before_they_are_multiplied(a_type, far):
    """1 << 62 values of two bytes are 0 bytes modulo 2^64, 1 << 61 of 8 rows the same: neither may pass for a small distance."""
    args = [P, P, 0, P, P, P, 0, P, P, 1 << 30]
    refused(RANGE, B.GroupedMatmul(8, 16, 32, 2, a_type=a_type, a_row=far), *args)
    refused(RANGE, B.GroupedMatmul(8, 16, 32, 2, a_type=a_type, b_row=far, b_expert=1 << 40), *args)
    refused(RANGE, B.GroupedMatmul(8, 9, 32, 1, a_type=a_type, b_row=far, b_expert=0), *args)
    if far > 1 << 59:
        refused(RANGE, B.GroupedMatmul(8, 16, 32, 2, a_type=a_type, b_expert=far), *args)


@pytest.mark.parametrize("S", [(1 << 30) + 1, (1 << 31) - (1 << 20), (1 << 31) - 1])
@pytest.mark.parametrize("x_type", ["f32", "f16", "bf16"])
def test_group_norm_refuses_positions_that_its_counters_pass(S, x_type):
    """Positions are counted in 32 bits, and a workgroup looks some beyond its own before it stops."""
    for y_type in (x_type, "e4m3"):
        op = B.GroupNorm(1, S, 1, 1, x_type=x_type, y_type=y_type)
        refused(RANGE, op, P, P, P, P, P, P, 1 << 30)
        with pytest.raises(B.SparseConvError) as e:
            op.workspace_size()
        assert e.value.status == RANGE
    assert B.GroupNorm(1, 1 << 30, 1, 1, x_type=x_type).workspace_size() > 0


def test_group_norm_compares_samples_without_overflow():
    """(S - 1) y_row + C beyond 64 bits is no distance that samples could have."""
    refused(SHAPE, B.GroupNorm(2, 5, 32, 4, y_strides=(1 << 40, 1 << 62)), P, P, P, P, 0, P, 1 << 20)
    refused(SHAPE, B.GroupNorm(2, 3, 32, 4, y_strides=(1 << 40, 1 << 62)), P, P, P, P, 0, P, 1 << 20)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("K", [(1 << 31) - 255, (1 << 31) - 15, (1 << 31) - 1])
def test_the_quantiser_refuses_columns_that_its_counters_pass(K, rows):
    """Columns are counted in 32 bits, up to the end of the last block and to the next multiple of 16."""
    refused(RANGE, B.BlockQuantizer(1, K, rows=rows), P, P, P)
    B.BlockQuantizer(0, (1 << 31) - 256, rows=rows).forward(0, 0, 0)


@pytest.mark.parametrize("shape,x_type,y_type", [((2, 3000, 48, 3), "f16", None), ((1, 500, 360, 30), "f16", "e4m3"), ((32, 3136, 256, 32), "bf16", "e4m3"), ((1, 5000, 7, 1), "f32", None)])
def test_group_norm_in_two_launches_refuses_workspaces_that_do_not_do(shape, x_type, y_type):
    op = B.GroupNorm(*shape, x_type=x_type, y_type=y_type)
    need = op.workspace_size()
    assert need > 0 and op.launch()["form"] == "norm two"
    for ws, size in ((0, 0), (0, need), (P, 0), (P, need - 1), (P + 4, need), (P + 8, need + 8)):
        refused(WORKSPACE, op, P, P, P, P, P, ws, size)
