"""The operators around a layer of experts on the GPU against their definitions in 64 bits (oracle/experts.py)."""
import numpy as np
import pytest
import torch

import test_experts_host as H
import test_operators_gpu as G
from oracle import experts as X
from paper_2112_15445_amd import binding as B

pytestmark = pytest.mark.gpu

T = G.T


def ints(*shape):
    """32-bit integers on the GPU that nothing has written yet."""
    return torch.full(shape, -77, dtype=torch.int32, device="cuda")


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


# -- router --------------------------------------------------------------------------------------

ROUTES = [  # tokens, experts, slots, elements between the end of a row and the next, elements before the first
    (1, 1, 1, 0, 0), (1, 64, 4, 0, 0), (2, 2, 2, 0, 1), (3, 7, 7, 1, 0), (17, 128, 8, 0, 0), (33, 129, 16, 3, 1), (16, 256, 16, 8, 8), (5, 100, 17, 0, 0), (9, 257, 3, 1, 0),
    (4, 512, 64, 0, 0), (6, 1000, 6, 0, 0), (2, 1024, 33, 5, 3), (3, 4096, 64, 0, 0), (5, 2049, 1, 3, 1), (250, 32, 2, 0, 0), (1025, 60, 4, 0, 0),
    (65, 121, 5, 0, 0), (65, 121, 6, 0, 0), (7, 12, 12, 0, 0), (40, 64, 16, 0, 0), (130, 300, 16, 3, 1), (9, 450, 5, 0, 0),         # keys compared, and sorted
]


def logits(T_, E, seed, kind="plain"):
    """Logits of a router; "ties": few distinct values; "out": many -inf and some NaN, rows that hold nothing else; "wide": far apart."""
    rng = np.random.default_rng(seed)
    x = 1.5 * rng.normal(size=(T_, E)) + rng.normal(size=E)
    if kind == "ties":
        x = np.round(x)
        x[:, ::3] = -0.0
    if kind == "out":
        x[rng.random((T_, E)) < 0.6] = -np.inf
        x[rng.random((T_, E)) < 0.1] = np.nan
        x[::5] = -np.inf
        x[1::7] = np.nan
    if kind == "wide":
        x = x * 40
        x[::2, 0] = -65504.0                                 # the lowest value of 16 bits, and all there is in some rows
        x[::4] = -65504.0
    return x


def run_route(x, top, x_type, pad=0, lead=0, bias=None, **kw):
    T_, E = x.shape
    _, xd = G.rows_of(x, x_type, E + pad, lead)
    ids, w = G.Out(T_, top, "f32"), G.Out(T_, top, "f32")
    bd = None if bias is None else dev(bias)
    B.ExpertRouter(T_, E, top, x_type=T[x_type], x_row=E + pad, **kw).forward(xd.data_ptr(), 0 if bd is None else bd.data_ptr(), ids.ptr, w.ptr, G.stream())
    torch.cuda.synchronize()
    ids.check_guard(), w.check_guard()
    return xd, ids.raw[:T_ * top].view(T_, top).cpu().numpy(), G.host(w.rows())


@pytest.mark.parametrize("x_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T_,E,top,pad,lead", ROUTES)
@pytest.mark.parametrize("kind", ["plain", "ties", "out", "wide"])
def test_route(T_, E, top, pad, lead, x_type, kind):
    x = logits(T_, E, T_ + 3 * E, kind)
    bias = None if kind == "wide" else (0.3 * np.random.default_rng(E).normal(size=E)).astype(np.float32)
    for score in ("softmax", "sigmoid"):
        for normalize in (False, True):
            for b in (None, bias):
                if b is not None and kind == "ties":
                    b = np.round(4 * b) / 4                  # (scores and biases that are equal stay equal)
                xd, ids, w = run_route(x, top, x_type, pad, lead, b, score=score, normalize=normalize, factor=2.5)
                ref_ids, ref, bound = X.route(G.host(xd), top, score, normalize, 2.5, b)
                what = (score, normalize, b is not None)
                if not np.array_equal(ids, ref_ids):         # scores that 64 bits do not tell apart may come in any order
                    assert b is not None, what
                    c = X.scores(G.host(xd), score) + b
                    for t, j in np.argwhere(ids != ref_ids):
                        assert ids[t, j] >= 0 and abs(c[t, ids[t, j]] - c[t, ref_ids[t, j]]) < 1e-14, (what, t, j)
                    continue
                G.assert_close(w, ref, bound, "f32", what)


def assert_chosen(ids, w, x, bias, score, normalize, factor):
    """What the header says of a choice with a bias: sums of score and bias whose first forty bits are alike may come in any order, and so may those that the score's own
    rounding (2^-51 of it) brings there; the numbers next to zero are 2^-1074 apart, twelve bits of them 2^-1062.  The weights are those of the ids that were chosen."""
    ref_ids = X.route(x, ids.shape[1], score, normalize, factor, bias)[0]
    s = X.scores(x, score)
    c = s + np.asarray(bias, np.float64)
    for t, j in np.argwhere(ids != ref_ids):
        g, r = ids[t, j], ref_ids[t, j]
        assert g >= 0 and abs(c[t, g] - c[t, r]) <= 2.0 ** -40 * max(abs(c[t, g]), abs(c[t, r])) + 2.0 ** -50 * max(s[t, g], s[t, r]) + 2.0 ** -1061, (t, j, ids[t], ref_ids[t])
    assert all(len(set(row[row >= 0])) == (row >= 0).sum() for row in ids)
    ref, bound = X.weights(x, ids, score, normalize, factor)
    G.assert_close(w, ref, bound, "f32", (score, normalize))


@pytest.mark.parametrize("x_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T_,E,top,pad,lead", ROUTES)
@pytest.mark.parametrize("kind", ["plain", "ties", "out", "wide"])
def test_route_with_a_bias(T_, E, top, pad, lead, x_type, kind):
    """Every kind of logits with a bias, and with one that is zero everywhere, where scores far below the largest still have an order."""
    x = logits(T_, E, T_ + 7 * E, kind)
    for bias in ((0.3 * np.random.default_rng(E).normal(size=E)).astype(np.float32), np.zeros(E, np.float32)):
        for score in ("softmax", "sigmoid"):
            for normalize in (False, True):
                xd, ids, w = run_route(x, top, x_type, pad, lead, bias, score=score, normalize=normalize, factor=2.5)
                assert_chosen(ids, w, G.host(xd), bias, score, normalize, 2.5)


@pytest.mark.parametrize("E,top", [(16, 16), (100, 16), (200, 15), (40, 20), (500, 30), (1000, 17), (3000, 64)])
def test_route_with_a_bias_orders_the_least_scores(E, top):
    """Scores that only 64 bits hold, e^-690 to e^-729, have their order, and those that are zero come behind them by rising number."""
    rng = np.random.default_rng(E)
    far = np.concatenate([[0], -690.0 - 3 * np.arange(14), -1000.0 - np.arange(E)])[:E]
    x = np.stack([far[rng.permutation(E)] for _ in range(9)])
    for score in ("softmax", "sigmoid"):
        ids = run_route(x, top, "f32", bias=np.zeros(E, np.float32), score=score)[1]
        assert np.array_equal(ids, X.route(x, top, score, bias=np.zeros(E))[0]), score


@pytest.mark.parametrize("x_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T_,E,top,pad,lead", ROUTES)
@pytest.mark.parametrize("kind", ["plain", "out", "wide"])
def test_route_backward(T_, E, top, pad, lead, x_type, kind):
    x = logits(T_, E, T_ + 5 * E, kind)
    rng = np.random.default_rng(E)
    _, xd = G.rows_of(x, x_type, E + pad, lead)
    ids = X.route(G.host(xd), top)[0]
    ids[::3, 0] = [E, -5, 1 << 30][T_ % 3]                   # ids of no expert
    if top > 1 and T_ > 1:
        ids[1, 1] = ids[1, 0]                                # the same expert twice
    dw = rng.normal(size=(T_, top)).astype(np.float32)
    dw[ids < 0] = np.nan                                     # what nobody reads
    idd, dwd = dev(ids, torch.int32), dev(dw)
    for score in ("softmax", "sigmoid"):
        for normalize in (False, True):
            dx = G.Out(T_, E, x_type, E + pad, lead)
            op = B.ExpertRouter(T_, E, top, x_type=T[x_type], x_row=E + pad, dx_row=E + pad, score=score, normalize=normalize, factor=1.5)
            op.backward(xd.data_ptr(), idd.data_ptr(), dwd.data_ptr(), dx.ptr, G.stream())
            torch.cuda.synchronize()
            ref, bound = X.route_backward(G.host(xd), ids, dw, score, normalize, 1.5)
            G.assert_close(G.host(dx.rows()), ref, bound, x_type, (score, normalize))
            dx.check_guard()


def test_route_of_infinite_logits_and_repeated_rows():
    """+inf is chosen first; a softmax of it is a NaN, as the formula has it, a sigmoid 1.  A row distance of 0 repeats the row."""
    x = torch.zeros(1, 40, device="cuda")
    x[0, 17] = float("inf")
    ids, w = B.route_experts_torch(x.expand(5, 40), 2)
    assert ids.tolist() == [[17, 0]] * 5 and bool(w.isnan().all())
    ids, w = B.route_experts_torch(x, 2, score="sigmoid")
    assert ids.tolist() == [[17, 0]] and w.tolist() == [[1.0, 0.5]]
    ids, w = B.route_experts_torch(torch.full((2, 40), -200.0, device="cuda"), 4, score="sigmoid", normalize=True)
    assert ids.tolist() == [[0, 1, 2, 3]] * 2 and w.tolist() == [[0.25] * 4] * 2


def test_route_backward_against_differences():
    """The gradient against central differences of the call's own weights, in 32 bits: steps of 2^-6 leave 2^-12 / 6 of the third derivative (at most 1)
    and 2 U 2^6 of the weights' roundings, some 1e-4 in all."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(6, 12, generator=g, device="cuda")
    dw = torch.randn(6, 3, generator=g, device="cuda")
    for score in ("softmax", "sigmoid"):
        for normalize in (False, True):
            ids, _ = B.route_experts_torch(x, 3, score, normalize)
            dx = B.route_experts_backward_torch(x, ids, dw, score, normalize)
            for e in range(12):
                ends = []
                for h in (2.0 ** -6, -2.0 ** -6):
                    y = x.clone()
                    y[:, e] += h
                    p = torch.softmax(y, 1) if score == "softmax" else torch.sigmoid(y)
                    w = p.gather(1, ids.long())
                    # the weights of these experts, whether or not the step changed their order
                    if normalize:
                        w = w / w.sum(1, keepdim=True)
                    there, got = B.route_experts_torch(y, 12, score)
                    own = torch.zeros_like(y).scatter_(1, there.long(), got).gather(1, ids.long())
                    own = own / own.sum(1, keepdim=True) if normalize else own
                    assert torch.allclose(own, w, rtol=1e-5)
                    ends.append((own * dw).sum(1))
                assert torch.allclose((ends[0] - ends[1]) * 2.0 ** 5, dx[:, e], atol=1e-3), (score, normalize, e)


def test_router_on_another_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    x = torch.randn(300, 96, device="cuda")
    ids, w = ints(300, 4), torch.zeros(300, 4, device="cuda")
    dw, dx = torch.randn(300, 4, device="cuda"), torch.zeros(300, 96, device="cuda")
    op = B.ExpertRouter(300, 96, 4, normalize=True)

    def run():
        op.forward(x.data_ptr(), 0, ids.data_ptr(), w.data_ptr(), s.cuda_stream)
        op.backward(x.data_ptr(), ids.data_ptr(), dw.data_ptr(), dx.data_ptr(), s.cuda_stream)

    inputs = [torch.randn(300, 96, device="cuda") for _ in range(3)]
    want = [B.route_experts_torch(v, 4, normalize=True) for v in inputs]
    grads = [B.route_experts_backward_torch(v, i, dw, normalize=True) for v, (i, _) in zip(inputs, want)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        x.copy_(inputs[0])
        run()
    s.synchronize()
    assert torch.equal(ids, want[0][0]) and torch.equal(w, want[0][1]) and torch.equal(dx, grads[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    for k in range(3):
        x.copy_(inputs[k])
        ids.fill_(-9), w.zero_(), dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, want[k][0]) and torch.equal(w, want[k][1]) and torch.equal(dx, grads[k])
        torch.zeros(1000, device="cuda").sum().item()


# -- rows sorted by expert -------------------------------------------------------------------------

SORTS = [  # tokens, slots, experts, how the ids are spread
    (1, 1, 1, "even"), (1, 8, 3, "even"), (8, 2, 16, "even"), (63, 1, 4096, "even"), (64, 1, 5, "one"), (65, 1, 5, "none"), (129, 7, 7, "out"), (1000, 3, 17, "skewed"),
    (1024, 1, 1024, "even"), (1025, 1, 1025, "out"), (4096, 2, 32, "skewed"), (4097, 2, 32, "skewed"), (8193, 1, 2, "even"), (5000, 64, 255, "out"), (3000, 5, 4096, "skewed"),
    (20000, 3, 256, "one"), (20001, 3, 257, "none"), (300000, 1, 3, "out"), (65536, 8, 256, "skewed"), (400001, 6, 100, "even"),
]


def choices(T_, top, E, kind):
    rng = np.random.default_rng(T_ + E)
    ids = rng.integers(0, E, size=(T_, top))
    if kind == "skewed":
        ids = np.minimum(rng.geometric(min(1.0, 4.0 / E), size=(T_, top)) - 1, E - 1)
    if kind == "one":
        ids[:] = E // 2
    if kind == "none":
        ids = rng.choice([-1, E, -2 ** 31, 2 ** 31 - 1], size=(T_, top))
    if kind == "out":
        ids = np.where(rng.random((T_, top)) < 0.3, rng.choice([-1, E, E + 1, -2 ** 31], size=(T_, top)), ids)
    return ids.astype(np.int32)


@pytest.mark.parametrize("T_,top,E,kind", SORTS)
def test_sort_by_expert(T_, top, E, kind):
    ids = choices(T_, top, E, kind)
    idd = dev(ids, torch.int32)
    off, index, position = G.Out(1, E + 1, "f32"), G.Out(1, T_ * top, "f32"), G.Out(T_, top, "f32")
    op = B.ExpertSort(T_, top, E)
    ws, wp, wn = G.workspace(op)
    for _ in range(2):                                       # (the workspace need not be clean)
        op.forward(idd.data_ptr(), off.ptr, index.ptr, position.ptr, wp, wn, G.stream())
    torch.cuda.synchronize()
    for got, want in zip((off, index, position), X.sort(ids, E)):
        got.check_guard()
        assert np.array_equal(got.rows().view(torch.int32).cpu().numpy().reshape(want.shape), want)
    assert int((ws[wn:] != 0xa5).sum()) == 0


def test_sort_of_many_slots_and_experts():
    """Thirty million slots of 4096 experts, 3663 chunks: against torch's stable sort."""
    g = torch.Generator(device="cuda").manual_seed(8)
    T_, top, E = 3750000, 8, 4096
    ids = torch.randint(-100, E + 50, (T_, top), generator=g, device="cuda", dtype=torch.int32)
    off, index, position = B.sort_by_expert_torch(ids, E)
    flat = torch.where((ids < 0) | (ids >= E), E, ids).reshape(-1)
    order = flat.sort(stable=True).indices
    n = int(off[E])
    assert torch.equal(off[1:].long(), torch.bincount(flat.long(), minlength=E + 1)[:E].cumsum(0)) and int(off[0]) == 0
    assert torch.equal(index[:n].long(), order[:n] // top) and bool((index[n:] == -1).all())
    want = torch.full((T_ * top,), -1, dtype=torch.int32, device="cuda")
    want[order[:n]] = torch.arange(n, dtype=torch.int32, device="cuda")
    assert torch.equal(position.view(-1), want)


def test_sort_of_no_tokens():
    off, index, position = B.sort_by_expert_torch(torch.empty(0, 3, dtype=torch.int32, device="cuda"), 4096)
    assert off.shape == (4097,) and not off.any() and index.shape == (0,) and position.shape == (0, 3)


def test_sort_on_another_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    for T_, top, E in ((700, 2, 40), (30000, 4, 300)):
        ids = ints(T_, top)
        off, index, position = ints(E + 1), ints(T_ * top), ints(T_, top)
        op = B.ExpertSort(T_, top, E)
        ws, wp, wn = G.workspace(op)

        def run():
            op.forward(ids.data_ptr(), off.data_ptr(), index.data_ptr(), position.data_ptr(), wp, wn, s.cuda_stream)

        inputs = [dev(choices(T_, top, E, kind), torch.int32) for kind in ("even", "out", "skewed")]
        want = [B.sort_by_expert_torch(v, E) for v in inputs]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            ids.copy_(inputs[1])
            run()
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((off, index, position), want[1]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run()
        for k in range(3):
            ids.copy_(inputs[k])
            off.fill_(-9), index.fill_(-9), position.fill_(-9)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((off, index, position), want[k]))
            torch.zeros(1000, device="cuda").sum().item()


# -- rows out and back -----------------------------------------------------------------------------

ROWS = [  # tokens, slots, columns, elements between the end of a row and the next, elements before the first
    (1, 1, 1, 0, 0), (1, 8, 16, 0, 0), (3, 2, 7, 1, 1), (65, 3, 30, 2, 0), (8, 2, 2048, 0, 0), (17, 4, 1100, 3, 1), (33, 1, 129, 0, 5), (5, 64, 520, 8, 8), (2, 3, 9001, 0, 0),
    (700, 2, 64, 0, 0), (300, 5, 8, 1, 0), (1030, 3, 603, 1, 0),
]
PAIRS = [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")]


def rows_case(T_, top, C, seed, extra=3):
    """(values [T top + extra, C], position) with some slots dropped and some whose rows do not exist."""
    rng = np.random.default_rng(seed)
    ids = rng.integers(-1, 6, size=(T_, top))
    position = X.sort(ids, 6)[2]
    bad = rng.random((T_, top)) < 0.1
    position = np.where(bad, rng.choice([T_ * top + extra, -1, 2 ** 31 - 1, -2 ** 31], size=(T_, top)), position).astype(np.int32)
    return rng, rng.normal(size=(T_ * top + extra, C)), position


@pytest.mark.parametrize("x_type", ["f32", "f16", "bf16", "e4m3"])
@pytest.mark.parametrize("T_,top,C,pad,lead", ROWS)
def test_gather_rows(T_, top, C, pad, lead, x_type):
    rng = np.random.default_rng(C)
    x = rng.normal(size=(T_, C))
    _, xd = G.rows_of(x, x_type, C + pad, lead)
    M = T_ * top
    index = rng.integers(-1, T_ + 1, size=M).astype(np.int32)
    index[:1] = 2 ** 31 - 1 if M > 1 else 0
    indexd = dev(index, torch.int32)
    y = G.Out(M, C, x_type, C + pad, lead)
    B.RowGather(M, C, T_, x_type=T[x_type], x_row=C + pad, y_row=C + pad).forward(xd.data_ptr(), indexd.data_ptr(), y.ptr, G.stream())
    torch.cuda.synchronize()
    live = (index >= 0) & (index < T_)
    want = np.where(live[:, None], G.host(xd)[np.where(live, index, 0)], 0)
    assert np.array_equal(G.host(y.rows()), want)
    y.check_guard()


@pytest.mark.parametrize("x_type,y_type", PAIRS)
@pytest.mark.parametrize("T_,top,C,pad,lead", ROWS)
def test_combine_rows(T_, top, C, pad, lead, x_type, y_type):
    rng, x, position = rows_case(T_, top, C, T_ + C)
    _, xd = G.rows_of(x, x_type, C + pad, lead)
    _, rd = G.rows_of(rng.normal(size=(T_, C)), y_type, C + pad, lead)
    live = (position >= 0) & (position < x.shape[0])
    w = np.where(live, rng.normal(size=(T_, top)), np.nan).astype(np.float32)       # (a slot without a row: whatever its weight)
    pd, wd = dev(position, torch.int32), dev(w)
    for weights in (w, None):
        for residual in (rd, None, "in place"):
            y = G.Out(T_, C, y_type, C + pad, lead)
            if residual is rd or residual is None:
                ptr, res = (0, None) if residual is None else (rd.data_ptr(), G.host(rd))
            else:
                y.rows().copy_(rd)
                ptr, res = y.ptr, G.host(rd)
            op = B.RowCombine(T_, top, C, x.shape[0], x_type=T[x_type], y_type=T[y_type], x_row=C + pad, y_row=C + pad, residual_row=C + pad)
            op.forward(xd.data_ptr(), pd.data_ptr(), 0 if weights is None else wd.data_ptr(), ptr, y.ptr, G.stream())
            torch.cuda.synchronize()
            ref, bound = X.combine(G.host(xd), position, weights, res)
            G.assert_close(G.host(y.rows()), ref, bound, y_type, (weights is None, residual is None))
            y.check_guard()


@pytest.mark.parametrize("x_type,y_type", PAIRS)
@pytest.mark.parametrize("T_,top,C,pad,lead", ROWS)
def test_combine_rows_backward(T_, top, C, pad, lead, x_type, y_type):
    rng, x, position = rows_case(T_, top, C, 2 * T_ + C)
    rows = x.shape[0]
    live = (position >= 0) & (position < rows)
    x[np.setdiff1d(np.arange(rows), position[live])] = np.nan                       # rows that no slot has are not read
    _, xd = G.rows_of(x, x_type, C + pad, lead)
    _, dyd = G.rows_of(rng.normal(size=(T_, C)), y_type, C + pad, lead)
    w = np.where(live, rng.normal(size=(T_, top)), np.nan).astype(np.float32)
    pd, wd = dev(position, torch.int32), dev(w)
    op = B.RowCombine(T_, top, C, rows, x_type=T[x_type], y_type=T[y_type], x_row=C + pad, y_row=C + pad, dx_row=C + pad)
    for weights in (w, None):
        dx, dw = G.Out(rows, C, x_type, C + pad, lead), G.Out(T_, top, "f32")
        op.backward(dyd.data_ptr(), xd.data_ptr(), pd.data_ptr(), 0 if weights is None else wd.data_ptr(), dx.ptr, dw.ptr, G.stream())
        torch.cuda.synchronize()
        ref, bound, ref_w, bound_w = X.combine_backward(G.host(dyd), np.nan_to_num(G.host(xd)), position, weights)
        at = np.sort(position[live])
        G.assert_close(G.host(dx.rows())[at], ref[at], bound[at], x_type, "dx")
        G.assert_close(G.host(dw.rows()), ref_w, bound_w, "f32", "dweights")
        dx.check_guard(written=at.tolist()), dw.check_guard()
        # either gradient alone
        only_x, only_w = G.Out(rows, C, x_type, C + pad, lead), G.Out(T_, top, "f32")
        op.backward(dyd.data_ptr(), 0, pd.data_ptr(), 0 if weights is None else wd.data_ptr(), only_x.ptr, 0, G.stream())
        op.backward(dyd.data_ptr(), xd.data_ptr(), pd.data_ptr(), 0 if weights is None else wd.data_ptr(), 0, only_w.ptr, G.stream())
        torch.cuda.synchronize()
        assert torch.equal(only_x.raw, dx.raw) and torch.equal(only_w.raw, dw.raw)


def test_gradient_of_rows_out_is_rows_back():
    """<gather(x), g> = <x, combine(g)>: the gradient of gather is combine without weights; and combine's against differences along a direction
    (it is linear: the difference of two calls is exact but for 32 bits)."""
    g = torch.Generator(device="cuda").manual_seed(0)
    ids = torch.randint(-1, 5, (40, 3), generator=g, device="cuda", dtype=torch.int32)
    off, index, position = B.sort_by_expert_torch(ids, 5)
    x, rows = torch.randn(40, 24, generator=g, device="cuda"), torch.randn(120, 24, generator=g, device="cuda")
    n = int(off[-1])
    rows[n:] = 0
    left = (B.gather_rows_torch(x, index).double() * rows.double()).sum()
    right = (x.double() * B.combine_rows_torch(rows, position).double()).sum()
    assert abs(float(left - right)) < 1e-4
    w, dy = torch.rand(40, 3, generator=g, device="cuda"), torch.randn(40, 24, generator=g, device="cuda")
    dx, dw = B.combine_rows_backward_torch(dy, rows, position, w)
    step_x, step_w = torch.randn(120, 24, generator=g, device="cuda"), torch.randn(40, 3, generator=g, device="cuda")
    step_x[n:] = 0
    for a, b, grad, step in ((rows + step_x, w, dx, step_x), (rows, w + step_w, dw, step_w)):
        change = ((B.combine_rows_torch(a, position, b).double() - B.combine_rows_torch(rows, position, w).double()) * dy.double()).sum()
        assert abs(float(change - (grad.double() * step.double()).sum())) < 1e-3


def test_rows_that_are_repeated_by_a_distance_of_0():
    """A matrix with one row for all, as a sum's gradient or a bias held as a base, is the matrix with that row copied."""
    g = torch.Generator(device="cuda").manual_seed(11)
    ids = torch.randint(-1, 4, (37, 3), generator=g, device="cuda", dtype=torch.int32)
    _, index, position = B.sort_by_expert_torch(ids, 4)
    for C in (50, 640):                                      # sixteen lanes a token and all of a workgroup's (gradients)
        one, w = torch.randn(1, C, generator=g, device="cuda"), torch.rand(37, 3, generator=g, device="cuda")
        rows = torch.randn(111, C, generator=g, device="cuda")
        for x, residual in ((one.expand(111, C), None), (rows, one.expand(37, C)), (one.expand(111, C), one.expand(37, C))):
            want = B.combine_rows_torch(x.contiguous(), position, w, None if residual is None else residual.contiguous())
            assert torch.equal(B.combine_rows_torch(x, position, w, residual), want)
            got, want = (B.combine_rows_backward_torch(dy, x, position, w) for dy in (one.expand(37, C), one.repeat(37, 1)))
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(B.gather_rows_torch(one.expand(37, C), index), B.gather_rows_torch(one.repeat(37, 1), index))
    for n, R in ((45, 16), (1700, 40)):                      # few rows, many
        x, a, b = torch.randn(n, 64, device="cuda").half(), torch.randn(2, R, 64, device="cuda").half(), torch.randn(2, 96, R, device="cuda").half()
        base, y = torch.randn(1, 96, device="cuda"), torch.full((n, 96), 7.0, device="cuda")
        off, index = torch.tensor([0, 20, n - 5], dtype=torch.int32, device="cuda"), torch.randperm(n, device="cuda").to(torch.int32)
        op = B.Adapters(n, 96, 64, R, 2, x_type="f16", y_type="f32", base_row=0)
        ws, wp, wn = G.workspace(op)
        op.forward(x.data_ptr(), index.data_ptr(), off.data_ptr(), a.data_ptr(), b.data_ptr(), 0, base.data_ptr(), y.data_ptr(), wp, wn, G.stream())
        assert torch.equal(y, B.adapters_torch(base.repeat(n, 1), x, a, b, off, index))


def test_two_graphs_that_share_a_workspace():
    """Replayed one after the other, in both orders: what one leaves in the workspace, the other does not take for its own."""
    s = torch.cuda.Stream()
    cases = []
    for T_, E, seed in ((9000, 40, 1), (9000, 7, 2)):
        g = torch.Generator(device="cuda").manual_seed(seed)
        ids = torch.randint(-1, E, (T_,), generator=g, device="cuda", dtype=torch.int32)
        x, a, b = (torch.randn(*shape, generator=g, device="cuda").half() for shape in ((T_, 72), (E, 40, 72), (E, 64, 40)))
        base, y = torch.randn(T_, 64, generator=g, device="cuda"), torch.empty(T_, 64, device="cuda")
        off, index, position = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (E + 1, T_, T_))
        sort, op = B.ExpertSort(T_, 1, E), B.Adapters(T_, 64, 72, 40, E, x_type="f16", y_type="f32")
        want = B.adapters_torch(base.clone(), x, a, b, *B.sort_by_expert_torch(ids, E)[:2])
        cases.append((ids, x, a, b, base, y, off, index, position, sort, op, want))
    n = max(max(c[9].workspace_size(), c[10].workspace_size()) for c in cases)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graphs = []
    for ids, x, a, b, base, y, off, index, position, sort, op, want in cases:
        assert sort.launch()["form"] == "sort chunks" and op.launch()["form"] == "adapters many"
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            sort.forward(ids.data_ptr(), off.data_ptr(), index.data_ptr(), position.data_ptr(), ws.data_ptr(), n, s.cuda_stream)
            op.forward(x.data_ptr(), index.data_ptr(), off.data_ptr(), a.data_ptr(), b.data_ptr(), 0, base.data_ptr(), y.data_ptr(), ws.data_ptr(), n, s.cuda_stream)
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (1, 1), (0, 0)):
        for c in cases:
            c[5].fill_(7)
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(cases[k][5], cases[k][11]) for k in order)
        torch.zeros(1000, device="cuda").sum().item()


def test_rows_of_nothing():
    x = torch.empty(0, 8, device="cuda")
    assert B.gather_rows_torch(x, ints(3)).tolist() == [[0.0] * 8] * 3
    assert B.combine_rows_torch(x, ints(2, 3), residual=torch.ones(2, 8, device="cuda")).tolist() == [[1.0] * 8] * 2
    dx, dw = B.combine_rows_backward_torch(torch.ones(2, 8, device="cuda"), x, ints(2, 3))
    assert dx.shape == (0, 8) and dw.tolist() == [[0.0] * 3] * 2
    assert B.gather_rows_torch(torch.ones(4, 8, device="cuda"), ints(0)).shape == (0, 8)


def test_combine_keeps_what_is_not_finite_in_its_token():
    x = torch.ones(6, 40, device="cuda")
    x[2, 5], x[3, 6] = float("nan"), float("inf")
    position = torch.tensor([[0, 1], [2, 3], [4, -1]], dtype=torch.int32, device="cuda")
    y = B.combine_rows_torch(x, position, torch.tensor([[1.0, 1.0], [1.0, 0.0], [2.0, float("nan")]], device="cuda"))
    assert y[0].eq(2).all() and y[2].eq(2).all() and y[1, 5].isnan() and y[1, 6].isnan() and y[1, :5].eq(1).all()


def test_rows_on_another_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    T_, top, C = 50, 3, 200
    ids = torch.randint(-1, 7, (T_, top), device="cuda", dtype=torch.int32)
    _, index, position = B.sort_by_expert_torch(ids, 7)
    x, w = torch.randn(T_, C, device="cuda"), torch.rand(T_, top, device="cuda")
    rows, y = torch.zeros(T_ * top, C, device="cuda"), torch.zeros(T_, C, device="cuda")
    dx, dw = torch.zeros(T_ * top, C, device="cuda"), torch.zeros(T_, top, device="cuda")
    out, back = B.RowGather(T_ * top, C, T_, x_type="f32"), B.RowCombine(T_, top, C, T_ * top, x_type="f32")

    def run():
        out.forward(x.data_ptr(), index.data_ptr(), rows.data_ptr(), s.cuda_stream)
        back.forward(rows.data_ptr(), position.data_ptr(), w.data_ptr(), 0, y.data_ptr(), s.cuda_stream)
        back.backward(y.data_ptr(), rows.data_ptr(), position.data_ptr(), w.data_ptr(), dx.data_ptr(), dw.data_ptr(), s.cuda_stream)

    inputs = [torch.randn(T_, C, device="cuda") for _ in range(3)]
    want = []
    for v in inputs:
        r = B.gather_rows_torch(v, index)
        z = B.combine_rows_torch(r, position, w)
        want.append((r, z, *B.combine_rows_backward_torch(z, r, position, w)))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        x.copy_(inputs[2])
        run()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((rows, y, dx, dw), want[2]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        run()
    for k in range(3):
        x.copy_(inputs[k])
        rows.zero_(), y.zero_(), dx.zero_(), dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((rows, y, dx, dw), want[k]))
        torch.zeros(1000, device="cuda").sum().item()


def test_rows_further_than_32_bits_reach():
    """Rows of 4 MB: the last ones of x, y and dx lie beyond 2^32 bytes."""
    M, C, row = 1100, 200, 1 << 20
    far = torch.zeros(M, row, device="cuda")                 # 4.6 GB
    x = torch.randn(M, C, device="cuda")
    far[:, :C] = x
    index = torch.arange(M - 1, -1, -1, dtype=torch.int32, device="cuda")
    assert torch.equal(B.gather_rows_torch(far[:, :C], index), x.flip(0))
    assert torch.equal(B.combine_rows_torch(far[:, :C], index[:, None]), x.flip(0))
    w, dy = torch.rand(M, 1, device="cuda"), torch.randn(M, C, device="cuda")
    want = B.combine_rows_backward_torch(dy, x, index[:, None], w)
    got = B.combine_rows_backward_torch(dy, far[:, :C], index[:, None], w)[1]
    assert torch.equal(got, want[1])
    st = G.stream()
    B.RowGather(M, C, M, x_type="f32", y_row=row).forward(want[0].data_ptr(), index.data_ptr(), far.data_ptr(), st)
    assert torch.equal(far[:, :C], want[0].flip(0))
    B.RowCombine(M, 1, C, M, x_type="f32", dx_row=row).backward(dy.data_ptr(), 0, index.data_ptr(), w.data_ptr(), far.data_ptr(), 0, st)
    assert torch.equal(far[:, :C], want[0])
    B.RowCombine(M, 1, C, M, x_type="f32", y_row=row).forward(x.data_ptr(), index.data_ptr(), 0, 0, far.data_ptr(), st)
    assert torch.equal(far[:, :C], x.flip(0))


@pytest.mark.parametrize("x_type,y_type", PAIRS)
@pytest.mark.parametrize("C,pad,lead", [(2056, 0, 0), (2053, 3, 1)])
def test_rows_of_large_results(C, pad, lead, x_type, y_type):
    """Results of more than 32 MiB, which go past the caches, against the same in parts, which stay in them: the same bits, and nothing between the rows."""
    size = 4 if y_type == "f32" else 2
    T_, top, step = (33 << 20) // (C * size) + 1, 2, 1000
    for rows, kind in ((T_, y_type), (2 * T_, x_type)):
        assert rows * C * (4 if kind == "f32" else 2) > 32 << 20
    g = torch.Generator(device="cuda").manual_seed(C)
    ids = torch.randint(-1, 5, (T_, top), generator=g, device="cuda", dtype=torch.int32)
    _, index, position = B.sort_by_expert_torch(ids, 5)
    made = lambda M, t: torch.randn(lead + M * (C + pad), generator=g, device="cuda").to(T[t])[lead:].view(M, C + pad)[:, :C]  # noqa: E731
    x, rows, residual, w = made(T_, x_type), made(T_ * top, x_type), made(T_, y_type), torch.rand(T_, top, generator=g, device="cuda")
    row = C + pad
    out = G.Out(T_ * top, C, x_type, row, lead)
    B.RowGather(T_ * top, C, T_, x_type=T[x_type], x_row=row, y_row=row).forward(x.data_ptr(), index.data_ptr(), out.ptr, G.stream())
    y = G.Out(T_, C, y_type, row, lead)
    op = B.RowCombine(T_, top, C, T_ * top, x_type=T[x_type], y_type=T[y_type], x_row=row, y_row=row, residual_row=row, dx_row=row)
    op.forward(rows.data_ptr(), position.data_ptr(), w.data_ptr(), residual.data_ptr(), y.ptr, G.stream())
    dx, dw = G.Out(T_ * top, C, x_type, row, lead), G.Out(T_, top, "f32")
    op.backward(residual.data_ptr(), rows.data_ptr(), position.data_ptr(), w.data_ptr(), dx.ptr, dw.ptr, G.stream())
    torch.cuda.synchronize()
    for t in range(0, T_ * top, step):
        assert torch.equal(out.rows()[t:t + step], B.gather_rows_torch(x, index[t:t + step]))
    taken = torch.zeros(T_ * top, dtype=torch.bool, device="cuda")
    for t in range(0, T_, step):
        p, part, some = position[t:t + step], w[t:t + step], slice(t, t + step)
        assert torch.equal(y.rows()[some], B.combine_rows_torch(rows, p, part, residual[some], dtype=T[y_type]))
        # (the gradient of a part of the tokens, with their own rows alone)
        there = p[p >= 0].long()
        own = torch.full_like(p, -1)
        own[p >= 0] = torch.arange(len(there), device="cuda", dtype=torch.int32)
        want = B.combine_rows_backward_torch(residual[some], rows[there], own, part)
        assert torch.equal(dx.rows()[there], want[0]) and torch.equal(dw.rows()[some], want[1])
        taken[there] = True
    out.check_guard(), y.check_guard(), dw.check_guard(), dx.check_guard(written=taken.nonzero()[:, 0].tolist())


# -- low-rank adapters ------------------------------------------------------------------------------

ADAPTERS = [  # rows of each adapter, rows without one, columns, summed values, rank
    ([1], 0, 16, 8, 1), ([1, 1, 0, 2], 0, 64, 64, 8), ([3, 0, 5], 2, 100, 72, 12), ([16, 17], 0, 333, 1100, 16), ([1] * 20, 3, 4096, 512, 16), ([40, 0, 90, 33], 7, 1000, 1100, 12),
    ([64, 65], 1, 256, 256, 32), ([70, 200], 0, 520, 264, 33), ([300], 0, 130, 1032, 64), ([5, 9], 0, 2048, 4096, 100), ([150, 100], 4, 600, 520, 128), ([2, 3], 0, 40, 136, 200),
    ([90, 60, 1], 0, 200, 300, 256), ([0, 0], 5, 64, 64, 8), ([1, 2] * 40, 0, 96, 40, 4), ([1400, 10], 0, 48, 520, 20),
    ([1500, 0, 70], 9, 200, 520, 33), ([2000, 40], 3, 70, 1100, 128), ([1600, 1], 0, 130, 136, 200), ([4000, 200], 5, 96, 72, 12), ([900] * 5, 0, 64, 40, 32),
    ([1700, 33], 0, 1030, 64, 64), ([2100, 5], 0, 40, 1100, 17), ([1100, 2], 1, 40, 1100, 250),
    ([8200, 0, 31], 3, 40, 1100, 20), ([8300, 1], 0, 72, 712, 64), ([8200, 8], 2, 34, 520, 100), ([8190, 5], 0, 40, 650, 256), ([16400, 7], 1, 40, 520, 9),
    ([300] * 55, 0, 64, 520, 33),
]


def adapter_rows(v, dtype, pad=0):
    """A stack of matrices on the GPU with rows on 16 bytes and NaN behind their ends."""
    E, rows, cols = v.shape
    row = -(-cols // 8) * 8 + pad
    full = torch.full((E, rows, row), float("nan"), device="cuda").to(T[dtype])
    full[:, :, :cols] = dev(v).to(T[dtype])
    return full


def run_adapters(counts, without, N, K, R, x_type, y_type, seed=0, use_index=True, in_place=False, odd=False, change=None):
    rng = np.random.default_rng(seed + N + K + R)
    E, M = len(counts), sum(counts)
    rows = M + without
    x, a, b = rng.normal(size=(rows, K)), rng.normal(size=(E, R, K)) * K ** -0.5, rng.normal(size=(E, N, R)) * R ** -0.5
    if change:
        change(x, a, b)
    xd, ad, bd = adapter_rows(x[None], x_type, 8 if odd else 0)[0], adapter_rows(a, x_type, 16 if odd else 0), adapter_rows(b, x_type, 8 if odd else 0)
    scale = rng.normal(size=E).astype(np.float32)
    order = rng.permutation(rows) if use_index else np.arange(rows)
    offsets = np.cumsum([0] + counts)
    groups = [order[lo:hi] for lo, hi in zip(offsets, offsets[1:])]
    base = rng.normal(size=(rows, N))
    lead = 3 if odd else 0
    _, based = G.rows_of(base, y_type, N + 5 * odd, lead)
    y = G.Out(rows, N, y_type, N + 5 * odd, lead)
    if in_place:
        y.rows().copy_(based)
        y.before = y.raw.clone()
    base_ptr = y.ptr if in_place else based.data_ptr()
    base_host = G.host(based)
    index, offd, sd = dev(order[:M], torch.int32), dev(offsets, torch.int32), dev(scale)
    op = B.Adapters(M, N, K, R, E, rows=rows, x_type=T[x_type], y_type=T[y_type], x_row=xd.stride(0), a_row=ad.stride(1), a_adapter=ad.stride(0), b_row=bd.stride(1),
                    b_adapter=bd.stride(0), base_row=N + 5 * odd, y_row=N + 5 * odd)
    ws, wp, wn = G.workspace(op)
    op.forward(xd.data_ptr(), index.data_ptr() if use_index else 0, offd.data_ptr(), ad.data_ptr(), bd.data_ptr(), sd.data_ptr(), base_ptr, y.ptr, wp, wn, G.stream())
    torch.cuda.synchronize()
    assert int((ws[wn:] != 0xa5).sum()) == 0
    xh, ah, bh = G.host(xd[:, :K]), G.host(ad[:, :, :K]), G.host(bd[:, :, :R])
    return y, *X.adapters(base_host, xh, ah, bh, groups, scale, x_type, y_type)


@pytest.mark.parametrize("x_type,y_type", PAIRS[1:])
@pytest.mark.parametrize("counts,without,N,K,R", ADAPTERS)
def test_adapters(counts, without, N, K, R, x_type, y_type):
    for i, kw in enumerate((dict(), dict(use_index=False, odd=True), dict(in_place=True), dict(odd=True, in_place=True))):
        y, ref, bound = run_adapters(counts, without, N, K, R, x_type, y_type, i, **kw)
        G.assert_close(G.host(y.rows()), ref, bound, y_type, kw)
        y.check_guard()


def test_both_forms_of_the_adapters_are_looked_at():
    forms = [(B.Adapters(sum(c), N, K, R, len(c)).launch()["form"], R) for c, _, N, K, R in ADAPTERS if sum(c)]
    ranks = {f: {max(16, 1 << (R - 1).bit_length()) for g, R in forms if g == f} for f, _ in forms}
    assert ranks == {"adapters few": {16, 32, 64, 128, 256}, "adapters many": {16, 32, 64, 128, 256}}
    assert {B.ExpertSort(t, k, e).launch()["form"] for t, k, e, _ in SORTS} == {"sort one", "sort chunks"}


@pytest.mark.parametrize("x_type", ["f16", "bf16"])
@pytest.mark.parametrize("more", [0, 1600])
def test_adapters_of_large_and_small_values(x_type, more):
    """What lies between the products is beyond the range of f16 on both sides, and differs by 2^20 within a row."""
    def change(x, a, b):
        x[:, :] = x * 200
        x[::2] *= 1e-3
        a[0] *= 400
        a[1] *= 2e-4
        a[:, ::2] *= 1e-3

    y, ref, bound = run_adapters([40 + more, 50], 0, 200, 512, 40, x_type, "f32", change=change)
    G.assert_close(G.host(y.rows()), ref, bound, "f32", "large and small")


@pytest.mark.parametrize("x_type,y_type", PAIRS[1:])
@pytest.mark.parametrize("counts", [[3, 0, 30], [1500, 0, 70]])
@pytest.mark.parametrize("R", [1, 9, 31, 65, 66, 82, 95, 96, 97, 127, 129, 161, 170, 191, 193, 223, 224, 225])
def test_adapters_ignore_what_lies_behind_the_ends_of_rows(R, counts, x_type, y_type):
    """NaN behind each row's end (adapter_rows), up to the next sixteen bytes and in the ranks that a form rounds R up to."""
    for kw in (dict(), dict(odd=True, in_place=True)):
        y, ref, bound = run_adapters(counts, 2, 72, 40, R, x_type, y_type, R, **kw)
        G.assert_close(G.host(y.rows()), ref, bound, y_type, kw)
        y.check_guard()


@pytest.mark.parametrize("y_type", ["bf16", "f32"])
@pytest.mark.parametrize("n,R", [(3, 8), (40, 104), (2100, 8), (1600, 40), (1600, 248)])
def test_adapters_of_a_first_product_near_the_end_of_the_range(n, R, y_type):
    """Sums between the largest bf16, (2 - 2^-7) 2^127, and the largest 32-bit float: finite, and so is what they become.  Products and sums of powers of two: 24 bits of
    the first product, of which the terms drop 2^-16 or 2^-24, times 2^-100."""
    x, a, b = torch.zeros(n, 16, device="cuda").bfloat16(), torch.zeros(2, R, 16, device="cuda").bfloat16(), torch.zeros(2, 70, R, device="cuda").bfloat16()
    x[:, 0], x[:, 1] = (2 - 2.0 ** -7) * 2.0 ** 127, 2.0 ** 119
    x[::2] *= -1
    a[:, :, 0] = 1
    a[:, :, 1] = torch.arange(R, device="cuda") % 3 / 2
    for r in range(R):
        b[:, r % 70, r] = 2.0 ** -100
    sign = torch.where(torch.arange(n, device="cuda") % 2 == 0, -1.0, 1.0)[:, None].double()
    got = B.adapters_torch(torch.zeros(n, 70, device="cuda", dtype=T[y_type]), x, a, b, torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda"))
    h = (2 - 2.0 ** -7) * 2.0 ** 127 + a[0, :, 1].double() * 2.0 ** 119
    want = sign * (h[None] @ b[0].double().t())
    # terms, the sum of up to four values in 32 bits, the result's own rounding
    bound = want.abs() * ((2.0 ** -16 + 2.0 ** -8 if y_type == "bf16" else 2.0 ** -23) + 8 * 2.0 ** -24)
    assert bool(got.isfinite().all()) and bool(((got.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("x_type,y_type", PAIRS[1:])
@pytest.mark.parametrize("counts,N,K,R", [([20], 72, 8200, 16), ([30, 9], 96, 4096, 256), ([700, 290], 2200, 264, 24), ([400, 400], 1900, 2056, 60), ([2, 0, 3], 200, 12296, 100), ([700], 2600, 1032, 200),
                                          ([1000, 1, 899], 1100, 2056, 17), ([1, 2], 40, 20000, 33)])
def test_adapters_of_few_rows_that_share_the_summed_dimension(counts, N, K, R, x_type, y_type):
    """Long sums, shared by 4, 8 and 16 workgroups, and waves with 3 and 4 times 32 columns (and both)."""
    assert B.Adapters(sum(counts), N, K, R, len(counts)).launch()["form"] == "adapters few"
    y, ref, bound = run_adapters(counts, 3, N, K, R, x_type, y_type, K)
    G.assert_close(G.host(y.rows()), ref, bound, y_type, "shared")
    y.check_guard()


@pytest.mark.parametrize("x_type", ["f16", "bf16"])
@pytest.mark.parametrize("n,R", [(40, 8), (40, 80), (2100, 24), (1600, 200)])
def test_adapters_keep_what_is_not_finite_in_b_in_its_column(n, R, x_type):
    x, a, b = (torch.randn(*shape, device="cuda").to(T[x_type]) for shape in ((n, 64), (2, R, 64), (2, 100, R)))
    off = torch.tensor([0, n // 2, n], dtype=torch.int32, device="cuda")
    want = B.adapters_torch(torch.zeros(n, 100, device="cuda"), x, a, b, off)
    b[0, 7, R - 1], b[0, 40, 0], b[1, 99, R // 2] = float("nan"), float("inf"), float("-inf")
    got = B.adapters_torch(torch.zeros(n, 100, device="cuda"), x, a, b, off)
    assert not got[:n // 2, [7, 40]].isfinite().any() and not got[n // 2:, 99].isfinite().any()
    got[:n // 2, [7, 40]], got[n // 2:, 99] = want[:n // 2, [7, 40]], want[n // 2:, 99]
    assert torch.equal(got, want)


@pytest.mark.parametrize("x_type,y_type", sorted(H.TERMS_KEPT))
@pytest.mark.parametrize("n,R", [(50, 16), (50, 24), (50, 56), (50, 120), (50, 248), (2100, 16), (2100, 24), (1100, 56), (1100, 120), (1100, 248)])
def test_adapters_first_product_keeps_its_bits(n, R, x_type, y_type):
    """A first product that is exact in 32 bits goes into the second one off by no more than is stated, 2^-24 (three bf16), 2^-16 (two), 2^-22 of the row's
    largest (two f16); nothing else rounds but the result."""
    x, a, b, scale, base, want, size = H.products_of_24_bits(n, R, 272, y_type)
    assert B.Adapters(n, 272, 16, R, 1, x_type=T[x_type], y_type=T[y_type]).launch()["form"] == ("adapters few" if n == 50 else "adapters many")
    xd, ad, bd = dev(x, T[x_type]), dev(a[None], T[x_type]), dev(b[None], T[x_type])
    got = B.adapters_torch(dev(base, T[y_type]), xd, ad, bd, torch.tensor([0, n], dtype=torch.int32, device="cuda"), scale=torch.full((1,), scale, device="cuda"))
    G.assert_close(G.host(got), want, H.TERMS_KEPT[x_type, y_type][1] * size, y_type, "terms")


@pytest.mark.parametrize("n,R", [(40, 8), (1600, 40)])
def test_adapters_keep_what_is_not_finite_in_its_row(n, R):
    x, a, b = torch.randn(n, 64, device="cuda").bfloat16(), torch.randn(2, R, 64, device="cuda").bfloat16(), torch.randn(2, 100, R, device="cuda").bfloat16()
    off = torch.tensor([0, 20, n], dtype=torch.int32, device="cuda")
    want = B.adapters_torch(torch.zeros(n, 100, device="cuda"), x, a, b, off)
    bad = x.clone()
    bad[3, 5], bad[25, 0] = float("nan"), float("inf")
    got = B.adapters_torch(torch.zeros(n, 100, device="cuda"), bad, a, b, off)
    rest = [i for i in range(n) if i not in (3, 25)]
    assert torch.equal(got[rest], want[rest]) and not got[3].isfinite().any() and not got[25].isfinite().any()


def test_adapters_with_indexes_and_offsets_that_are_out_of_range():
    x, a, b = torch.randn(30, 64, device="cuda").half(), torch.randn(3, 16, 64, device="cuda").half(), torch.randn(3, 80, 16, device="cuda").half()
    off = torch.tensor([-5, 4, 4, 1 << 30], dtype=torch.int32, device="cuda")            # clamped: 0 .. 4, none, 4 .. 12
    index = torch.tensor([29, -1, 3, 30, 7, 0, 2 ** 31 - 1, -2 ** 31, 5, 6, 28, 1], dtype=torch.int32, device="cuda")
    y = torch.full((30, 80), 2.0, device="cuda")
    got = B.adapters_torch(y.clone(), x, a, b, off, index)
    for e, named in ((0, [29, 3]), (2, [7, 0, 5, 6, 28, 1])):
        for t in named:
            want = B.adapters_torch(y[:1].clone(), x[t:t + 1], a[e:e + 1], b[e:e + 1], torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
            assert torch.allclose(got[t], want[0], rtol=1e-5, atol=1e-5)
    others = [t for t in range(30) if t not in (29, 3, 7, 0, 5, 6, 28, 1)]
    assert bool((got[others] == 2.0).all())


def test_adapters_rows_that_no_group_names_keep_base():
    """Whatever the workspace holds: places of an earlier call with other groups, and every number a stale place can be."""
    for rows, R in ((200, 8), (4200, 64)):
        keeps_base(rows, 64, 72, R)


def keeps_base(rows, K, N, R):
    x, a, b = torch.randn(rows, K, device="cuda").half(), torch.randn(3, R, K, device="cuda").half(), torch.randn(3, N, R, device="cuda").half()
    base = torch.randn(rows, N, device="cuda")
    index = torch.randperm(rows, device="cuda").to(torch.int32)
    op = B.Adapters(rows, N, K, R, 3, x_type="f16", y_type="f32")
    ws = torch.zeros(op.workspace_size() // 4, dtype=torch.int32, device="cuda")
    for fill, bounds in ((None, [0, 90, 90, rows]), (None, [30, 40, 60, 100]), (0, [0, 0, 50, 50]), (-1, [rows - 1, rows - 1, rows - 1, rows]), (199, [150, 200, 200, 200]), (2 ** 31 - 1, [0, 0, 0, 0]), (None, [0, 1, 2, 3])):
        off = torch.tensor(bounds, dtype=torch.int32, device="cuda")
        if fill is not None:
            ws.fill_(fill)
        for i in (index, None):
            y = torch.full((rows, N), 7.0, device="cuda")
            op.forward(x.data_ptr(), 0 if i is None else i.data_ptr(), off.data_ptr(), a.data_ptr(), b.data_ptr(), 0, base.data_ptr(), y.data_ptr(), ws.data_ptr(), 4 * ws.numel(), G.stream())
            want = B.adapters_torch(base.clone(), x, a, b, off, i)
            assert torch.equal(y, want), (fill, bounds)
            named = torch.arange(rows, device="cuda")[bounds[0]:bounds[3]] if i is None else index[bounds[0]:bounds[3]].long()
            rest = torch.ones(rows, dtype=torch.bool, device="cuda")
            rest[named] = False
            assert torch.equal(y[rest], base[rest]) and (named.numel() == 0 or not torch.equal(y[named], base[named]))
    y = torch.full((rows, N), 7.0, device="cuda")             # no groups at all
    B.Adapters(0, N, K, R, 3, rows=rows, x_type="f16", y_type="f32").forward(0, 0, 0, 0, 0, 0, base.data_ptr(), y.data_ptr(), 0, 0, G.stream())
    assert torch.equal(y, base)


def test_adapters_of_nothing():
    x, a, b = torch.empty(0, 64, device="cuda").half(), torch.randn(3, 16, 64, device="cuda").half(), torch.randn(3, 80, 16, device="cuda").half()
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert B.adapters_torch(torch.empty(0, 80, device="cuda"), x, a, b, off).shape == (0, 80)
    assert B.adapters_torch(torch.empty(0, 80, device="cuda"), x, a, b, off, ints(3)).shape == (0, 80)


def test_adapters_twice_on_another_stream_and_in_a_graph():
    s = torch.cuda.Stream()
    for T_, E, R, K, N in ((9, 4, 16, 1024, 640), (500, 3, 64, 512, 640), (1800, 3, 64, 512, 640)):
        ids = torch.randint(-1, E, (T_,), device="cuda", dtype=torch.int32)
        off, index, _ = B.sort_by_expert_torch(ids, E)
        x, a, b = torch.randn(T_, K, device="cuda").bfloat16(), torch.randn(E, R, K, device="cuda").bfloat16(), torch.randn(E, N, R, device="cuda").bfloat16()
        base, y = torch.randn(T_, N, device="cuda"), torch.zeros(T_, N, device="cuda")
        op = B.Adapters(T_, N, K, R, E, y_type="f32")
        ws, wp, wn = G.workspace(op)

        def run():
            op.forward(x.data_ptr(), index.data_ptr(), off.data_ptr(), a.data_ptr(), b.data_ptr(), 0, base.data_ptr(), y.data_ptr(), wp, wn, s.cuda_stream)

        inputs = [torch.randn(T_, K, device="cuda").bfloat16() for _ in range(3)]
        live = (ids >= 0)[:, None]
        want = [B.adapters_torch(base.clone(), v, a, b, off, index) for v in inputs]
        assert all(torch.equal(w[~live[:, 0]], base[~live[:, 0]]) for w in want)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            x.copy_(inputs[2])
            run()
        s.synchronize()
        assert torch.equal(y, want[2])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run()
        for k in range(3):
            x.copy_(inputs[k])
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want[k])
            torch.zeros(1000, device="cuda").sum().item()


def test_router_and_adapters_further_than_32_bits_reach():
    """Rows of 4 MB (of x of the adapters: just below): the last logits, gradients, rows of x, base and y lie beyond 2^32 bytes."""
    M, E, row = 1100, 48, 1 << 20
    far = torch.zeros(M, row, device="cuda")                 # 4.6 GB
    logits, dw = torch.randn(M, E, device="cuda"), torch.randn(M, 3, device="cuda")
    far[:, :E] = logits
    ids, w = B.route_experts_torch(logits, 3)
    far_ids, far_w = B.route_experts_torch(far[:, :E], 3)
    assert torch.equal(ids, far_ids) and torch.equal(w, far_w)
    want = B.route_experts_backward_torch(logits, ids, dw)
    B.ExpertRouter(M, E, 3, x_row=row, dx_row=row).backward(far.data_ptr(), ids.data_ptr(), dw.data_ptr(), far[:, 64:].data_ptr(), G.stream())
    assert torch.equal(far[:, 64:64 + E], want)
    for rows in (M, 1700):                                   # few rows, many
        K, N, R, wide = 96, 80, 40, (1 << 21) - 8
        x, a, b = torch.randn(rows, K, device="cuda").half(), torch.randn(2, R, K, device="cuda").half(), torch.randn(2, N, R, device="cuda").half()
        off = torch.tensor([0, 30, rows], dtype=torch.int32, device="cuda")
        base = torch.randn(rows, N, device="cuda")
        want = B.adapters_torch(base.clone(), x, a, b, off)
        del far
        far = torch.zeros(rows, wide, dtype=torch.float16, device="cuda")
        far[:, :K] = x
        assert torch.equal(B.adapters_torch(base.clone(), far[:, :K], a, b, off), want)
        del far
        far = torch.zeros(rows, row, device="cuda")
        far[:, :N] = base
        assert torch.equal(B.adapters_torch(far[:, :N], x, a, b, off), want)


# -- all of them together ---------------------------------------------------------------------------

def test_a_layer_of_experts_and_its_gradients():
    """Router, sort, rows out, products by expert, rows back with a residual, and the gradients back through all of it, in 32 bits (the products and their gradients
    torch's), against autograd in 64 bits.  A chain of sums of up to 96 values in 32 bits: 1e-5 of the largest is some hundred roundings."""
    g = torch.Generator(device="cuda").manual_seed(4)
    T_, E, top, C = 300, 6, 2, 96
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, router, expert, dy = rand(T_, C), rand(E, C) * C ** -0.5, rand(E, C, C) * C ** -0.5, rand(T_, C)

    logits = x @ router.t()
    ids, w = B.route_experts_torch(logits, top, normalize=True)
    offsets, index, position = B.sort_by_expert_torch(ids, E)
    bounds = offsets.tolist()
    assert bounds[-1] == T_ * top
    rows = B.gather_rows_torch(x, index)
    parts = [slice(lo, hi) for lo, hi in zip(bounds, bounds[1:])]
    h = torch.cat([rows[p] @ expert[e].t() for e, p in enumerate(parts)])
    y = B.combine_rows_torch(h, position, w, residual=x)

    dh, dw = B.combine_rows_backward_torch(dy, h, position, w)
    drows = torch.cat([dh[p] @ expert[e] for e, p in enumerate(parts)])
    dexpert = torch.stack([dh[p].t() @ rows[p] for p in parts])
    dlogits = B.route_experts_backward_torch(logits, ids, dw, normalize=True)
    dx = B.combine_rows_torch(drows, position, residual=dy) + dlogits @ router
    drouter = dlogits.t() @ x

    X64, R64, E64 = (v.double().requires_grad_() for v in (x, router, expert))
    p = torch.softmax(X64 @ R64.t(), 1).gather(1, ids.long())
    p = p / p.sum(1, keepdim=True)
    each = torch.matmul(E64[ids.reshape(-1).long()], X64.repeat_interleave(top, 0)[:, :, None])[:, :, 0].view(T_, top, C)
    want = X64 + (each * p[:, :, None]).sum(1)
    want.backward(dy.double())
    for got, ref in ((y, want.detach()), (dx, X64.grad), (drouter, R64.grad), (dexpert, E64.grad)):
        assert float((got.double() - ref).abs().max()) < 1e-5 * max(1.0, float(ref.abs().max())), got.shape


def test_experts_in_16_bits_as_they_are_served():
    """The same layer forward through the library's products, tokens closed to most experts and some to all of them, in one graph."""
    g = torch.Generator(device="cuda").manual_seed(5)
    T_, E, top, C, H = 64, 8, 3, 128, 192
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    first, second = (rand(E, H, C) * C ** -0.5).half(), (rand(E, C, H) * H ** -0.5).half()
    x, logits = rand(T_, C).half(), rand(T_, E)
    logits[rand(T_, E) < 0.3] = float("-inf")
    logits[::9] = float("-inf")
    s = torch.cuda.Stream()

    def layer():
        ids, w = B.route_experts_torch(logits, top, normalize=True)
        offsets, index, position = B.sort_by_expert_torch(ids, E)
        h = B.matmul_grouped_torch(x, first, offsets, index=index, act="silu")
        return ids, w, B.combine_rows_torch(B.matmul_grouped_torch(h, second, offsets), position, w, residual=x)

    with torch.cuda.stream(s):
        layer()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        ids, w, y = layer()
    for k in range(3):
        x.copy_(rand(T_, C).half())
        graph.replay()
        torch.cuda.synchronize()
        e_ids, e_w, e_y = layer()
        assert torch.equal(ids, e_ids) and torch.equal(w, e_w) and torch.equal(y, e_y)
        ref = x.double()
        for j in range(top):
            live = ids[:, j] >= 0
            z = torch.matmul(first.double()[ids[live, j].long()], x.double()[live][:, :, None])[:, :, 0]
            z = torch.nn.functional.silu(z).half().double()
            ref[live] += w[live, j].double()[:, None] * torch.matmul(second.double()[ids[live, j].long()], z[:, :, None])[:, :, 0]
        assert torch.equal(y[::9], x[::9])                   # nothing is added where no expert is left
        # what is rounded to f16: the first layer (its own rounding may fall the other way), the second, the sum: 2^-11 each of values of up to some 8
        assert float((y.double() - ref).abs().max()) < 4 * 8 * 2.0 ** -11
        torch.zeros(1000, device="cuda").sum().item()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_the_example_rounds_once(dtype):
    """The block of examples/channels_last_experts.py adds the experts' 32-bit rows to its input in 32 bits and rounds the sum, nothing before."""
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("example", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "channels_last_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    block = m.Block(192)
    x = torch.randn(2, 63, 192, device="cuda").to(T[dtype])
    out, (weights, offsets, index, position) = block.forward(x)
    q, scale = B.group_norm_torch(x, block.groups, block.gamma, block.beta, act="silu", codes=True)
    h = B.matmul_grouped_torch(q, block.first_q[0], offsets, scale, block.first_q[1], index=index, bias=block.bias, act="silu")
    hq, h_scale = B.quantize_blocks_torch(h)
    y = B.matmul_grouped_torch(hq, block.second_q[0], offsets, h_scale, block.second_q[1], dtype=torch.float32)
    ref, bound = X.combine(G.host(y), position.cpu().numpy(), G.host(weights), G.host(x).reshape(-1, 192))
    assert out.dtype == x.dtype
    G.assert_close(G.host(out).reshape(-1, 192), ref, bound, dtype, "block")


def test_adapters_beside_a_shared_projection():
    """A projection for all tokens (the products by expert with one expert), the adapters of four requests on top, some tokens without one."""
    g = torch.Generator(device="cuda").manual_seed(6)
    for T_ in (1, 5, 90, 2000):
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
        x, weight, a, b = rand(T_, 256), rand(1, 320, 256) / 16, rand(4, 40, 256) / 16, rand(4, 320, 40) / 6
        scale = torch.tensor([0.5, 1.0, 2.0, -1.0], device="cuda")
        ids = torch.randint(-1, 4, (T_,), generator=g, device="cuda", dtype=torch.int32)
        everything = torch.tensor([0, T_], dtype=torch.int32, device="cuda")
        offsets, index, _ = B.sort_by_expert_torch(ids, 4)
        y = B.matmul_grouped_torch(x, weight, everything, dtype=torch.float32)
        got = B.adapters_torch(y, x, a, b, offsets, index, scale)
        ref = x.double() @ weight[0].double().t()
        for e in range(4):
            rows = ids == e
            ref[rows] += float(scale[e]) * (x[rows].double() @ a[e].double().t()) @ b[e].double().t()
        assert float((got.double() - ref).abs().max()) < 1e-4    # 256 + 40 products in 32 bits, and what three bf16 terms leave: 2^-23
