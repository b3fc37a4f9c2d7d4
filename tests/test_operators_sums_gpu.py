"""Products of codes with 16-bit results on the GPU: all elements together against what the 8-bit cores' way to add leaves, and no more."""
import numpy as np
import pytest
import torch

import test_operators_gpu as T
from oracle import operators as O
from paper_2112_15445_amd import binding as B
from test_operators_forms_gpu import PRODUCTS
from test_operators_sums_host import KINDS, operands

pytestmark = pytest.mark.gpu


def put_codes(ca, cb, sa, sb):
    """The operands on the GPU, rows on 16 bytes."""
    def up(c):
        q = B.empty_codes(*c.shape)
        q.view(torch.uint8).copy_(torch.from_numpy(c).to(torch.float8_e4m3fn).view(torch.uint8))
        return q
    return up(ca), up(cb), torch.from_numpy(sa).cuda(), torch.from_numpy(sb).cuda()


@pytest.mark.parametrize("y_type", ["f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("form", list(PRODUCTS))
def test_products_of_codes_as_a_whole(form, kind, y_type):
    """All elements of some rows together against the definition, allowed what the 8-bit cores' way to add leaves; large values among
    small ones included.  (Element by element the bound of O.product has to allow the worst case, a hundred times as much.)"""
    M, N, K = PRODUCTS[form]
    ca, sa, cb, sb = operands(kind, M, N, K, seed=len(form))
    qa, qb, asc, bsc = put_codes(ca, cb, sa, sb)
    y = B.matmul_blocks_torch(qa, asc, qb, bsc, dtype=T.T[y_type])
    at = np.unique(np.linspace(0, M - 1, 40).astype(int))
    columns = np.unique(np.concatenate([np.linspace(0, N - 1, 480).astype(int), [127, 128, 255, 256, N - 1]]))
    sel = (ca[at], sa[at], cb[columns])
    scale = sb[columns // 128]                                # (of single columns)
    ref = O.values(sel[0], sel[1], 1) @ (sel[2].astype(np.float64) * scale.astype(np.float64)[:, np.arange(K) // 128]).T
    model = core_sums_of_columns(*sel, scale)
    off = O.aggregate(T.host(y)[at][:, columns], ref, model, y_type)
    print(form, kind, y_type, "share of the allowance", off, flush=True)
    assert off <= 1


def core_sums_of_columns(ca, sa, cb, scale):
    """O.core_sums for columns picked from several blocks, whose scales are [columns, blocks of K]."""
    out = np.zeros((ca.shape[0], cb.shape[0]))
    for first in range(0, cb.shape[0], 128):
        part = slice(first, first + 128)
        for n in range(scale.shape[1]):
            k = slice(n * 128, (n + 1) * 128)
            out[:, part] += O.core_sums(ca[:, k], np.ones((ca.shape[0], 1)), cb[part, k], np.ones((1, 1))) * sa[:, n:n + 1].astype(np.float64) * scale[part, n].astype(np.float64)
    return out


@pytest.mark.parametrize("y_type", ["f16", "bf16"])
@pytest.mark.parametrize("counts,N,K", [([0, 30, 200, 2], 700, 520), ([900, 0, 1200, 1197], 2060, 640)])
def test_products_of_codes_by_expert_as_a_whole(counts, N, K, y_type):
    """The last expert's rows, picked by an index."""
    M, E = sum(counts), len(counts)
    parts = [operands("outliers", 300, N, K, seed=e) for e in range(E)]
    ca, sa = parts[0][:2]
    index = np.random.default_rng(3).integers(0, 300, size=M).astype(np.int32)
    qa, _, asc, _ = put_codes(ca, parts[0][2], sa, parts[0][3])
    qb = B.empty_codes(E, N, K)
    for e in range(E):
        qb[e].view(torch.uint8).copy_(torch.from_numpy(parts[e][2]).to(torch.float8_e4m3fn).view(torch.uint8))
    bsc = torch.from_numpy(np.stack([p[3] for p in parts])).cuda()
    off = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")
    y = B.matmul_grouped_torch(qa, qb, off, asc, bsc, index=torch.from_numpy(index).cuda(), dtype=T.T[y_type])
    e = 2
    at = np.arange(sum(counts[:e]), sum(counts[:e + 1]))[:: max(1, counts[e] // 40)]
    cb, sb = parts[e][2:]
    pick = index[at]
    ref = O.values(ca[pick], sa[pick], 1) @ O.values(cb, sb, 128).T
    model = O.core_sums(ca[pick], sa[pick], cb, sb)
    assert O.aggregate(T.host(y)[at], ref, model, y_type) <= 1
