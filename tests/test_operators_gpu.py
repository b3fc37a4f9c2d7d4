"""The operators of channels-last blocks on the GPU against their definitions in 64 bits (oracle/operators.py)."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from paper_2112_15445_amd import binding as B

pytestmark = pytest.mark.gpu

T = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
NAN_CODE = 0x7f


def stream():
    return torch.cuda.current_stream().cuda_stream


def host(t):
    return t.detach().float().cpu().numpy()


def workspace(op):
    n = op.workspace_size()
    ws = torch.full((max(n, 16),), 0xa5, dtype=torch.uint8, device="cuda")
    return ws, ws.data_ptr(), n


def rows_of(values, dtype, row, lead=0):
    """`values` [M, K] on the GPU in rows `row` elements apart, `lead` elements into an allocation filled with NaN."""
    M, K = values.shape
    buf = torch.full((lead + M * row + 16,), float("nan"), device="cuda").to(T[dtype])
    view = buf[lead:lead + M * row].view(M, row)
    view[:, :K] = torch.from_numpy(np.ascontiguousarray(values)).cuda().to(T[dtype])
    return buf, view[:, :K]


class Out:
    """M rows of N elements, `row` apart, between guard bytes that nothing may write."""

    def __init__(self, M, N, dtype, row=None, lead=0):
        row = N if row is None else row
        self.raw = torch.full((lead + M * row + 64,), 1, dtype=torch.int32 if dtype == "f32" else torch.int8 if dtype == "e4m3" else torch.int16, device="cuda")
        self.raw.view(torch.uint8).fill_(0x5b)
        self.before = self.raw.clone()
        self.M, self.N, self.row, self.lead, self.dtype = M, N, row, lead, dtype
        self.ptr = self.raw.data_ptr() + lead * self.raw.element_size()

    def rows(self):
        return self.raw[self.lead:self.lead + self.M * self.row].view(self.M, self.row).view(T[self.dtype])[:, :self.N]

    def check_guard(self, written=None, pad=0):
        """Everything but the N + pad elements of the rows in `written` is as it was."""
        mask = torch.zeros_like(self.raw, dtype=torch.bool)
        part = mask[self.lead:self.lead + self.M * self.row].view(self.M, self.row)
        for m in range(self.M) if written is None else written:
            part[m, :self.N + pad] = True
        assert torch.equal(self.raw[~mask], self.before[~mask])


def assert_close(y, ref, bound, ytype, what):
    over, at, got, want = O.excess(y, ref, bound, ytype)
    assert over <= 0, f"{what}: element {at}: {got!r} for {want!r}, {over:.3e} outside what is allowed"


# -- quantisation --------------------------------------------------------------------------------

@pytest.mark.parametrize("x_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("M,K,pad,lead", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 3, 1), (128, 128, 0, 0), (129, 1100, 4, 0),
                                          (130, 100, 28, 8), (257, 256, 0, 0), (5, 2048, 0, 0), (300, 384, 1, 0), (64, 8192, 0, 0)])
def test_quantize_blocks_bit_for_bit(x_type, rows, M, K, pad, lead):
    rng = np.random.default_rng(M * 7 + K)
    x = (rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, 1)))).astype(np.float32)
    x[0, :min(K, 5)] = [0.0, -0.0, 1e-30, -2.0, 448.0][:min(K, 5)]
    if M > 2:
        x[2] = 0.0                                            # blocks without a value
    _, xd = rows_of(x, x_type, K + pad, lead)
    q_row = -(-K // 16) * 16 + 16 * (pad > 0)
    kb = -(-K // 128)
    q = Out(M, K, "e4m3", q_row)
    s = Out(-(-M // rows), kb, "f32", kb + (pad > 0))
    op = B.BlockQuantizer(M, K, rows=rows, x_type=T[x_type], x_row=K + pad, q_row=q_row, scale_row=kb + (pad > 0))
    op.forward(xd.data_ptr(), q.ptr, s.ptr, stream())
    torch.cuda.synchronize()
    code, scale = O.quantize(host(xd), rows)
    assert np.array_equal(host(s.rows()), scale)
    assert np.array_equal(host(q.rows()), code)
    fill = -K % 16                                            # zero codes up to the next multiple of 16
    whole = q.raw.view(torch.uint8)[:M * q_row].view(M, q_row)
    assert int(whole[:, K:K + fill].abs().max() if fill else 0) == 0
    q.check_guard(pad=fill)
    s.check_guard()


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_blocks_of_what_is_not_finite_or_tiny(rows):
    x = np.ones((4, 512), np.float32)
    x[1, 3] = np.nan
    x[1, 4] = 7.0
    x[2, 128:256] = np.nan
    x[3, 300] = np.inf
    x[3, 301] = -3.0
    x[:, 384:] = 1e-38                                        # below the smallest magnitude that scales a block
    _, xd = rows_of(x, "f32", 512)
    q, s = Out(4, 512, "e4m3"), Out(4 if rows == 1 else 1, 4, "f32")
    B.BlockQuantizer(4, 512, rows=rows, x_type="f32").forward(xd.data_ptr(), q.ptr, s.ptr, stream())
    torch.cuda.synchronize()
    code, scale = O.quantize(x, rows)
    got = host(q.rows())
    assert np.array_equal(host(s.rows()), scale)
    assert np.array_equal(np.isnan(got), np.isnan(code))
    assert np.array_equal(got[~np.isnan(got)], code[~np.isnan(code)])
    assert np.isnan(got[1, 3]) and np.isnan(got[3, 300]) and not np.isnan(got[3, 301])


# -- group norm ----------------------------------------------------------------------------------

NORM_SHAPES = [  # N, S, C, G, extra elements between positions, elements before the first
    (1, 1, 32, 32, 0, 0), (1, 1, 64, 8, 0, 0), (2, 49, 2048, 32, 0, 0), (3, 7, 100, 10, 0, 0), (2, 37, 360, 30, 8, 0),
    (1, 837, 360, 30, 0, 0), (2, 64, 96, 1, 3, 1), (1, 3000, 64, 32, 0, 0), (5, 16, 30, 30, 2, 0), (1, 5000, 7, 1, 0, 1),
    (2, 3136, 256, 32, 0, 0), (1, 196, 1024, 16, 8, 8), (33, 5, 24, 3, 0, 0),
    (2, 4, 844, 1, 0, 0), (3, 1, 7, 7, 0, 0), (2, 300, 130, 13, 0, 0), (2, 90, 520, 4, 3, 1), (1, 1000, 52, 2, 0, 0), (2, 20, 2040, 1020, 0, 0), (1, 2, 6000, 3000, 0, 0),
    (1, 700, 5000, 2, 0, 0), (1, 900, 700, 700, 0, 0),
]


def norm_inputs(N, S, C, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(N, S, C)) * (0.5 + rng.random(C)) + 2.0 * rng.normal(size=C)
    return x, (1 + 0.2 * rng.normal(size=C)).astype(np.float32), (0.2 * rng.normal(size=C)).astype(np.float32)


def run_norm(x, G, gamma, beta, x_type, y_type, kind, pad=0, lead=0, y_pad=0, eps=1e-5):
    N, S, C = x.shape
    _, xd = rows_of(x.reshape(N * S, C), x_type, C + pad, lead)
    codes = y_type == "e4m3"
    row = -(-C // 16) * 16 if codes else C + y_pad
    y = Out(N * S, C, y_type, row)
    kb = -(-C // 128)
    ys = Out(N * S, kb, "f32") if codes else None
    gd = None if gamma is None else torch.from_numpy(gamma).cuda()
    bd = None if beta is None else torch.from_numpy(beta).cuda()
    op = B.GroupNorm(N, S, C, G, eps=eps, act=kind, x_type=T[x_type], y_type=T[y_type], x_strides=(S * (C + pad), C + pad), y_strides=(S * row, row))
    ws, wp, wn = workspace(op)
    op.forward(xd.data_ptr(), 0 if gd is None else gd.data_ptr(), 0 if bd is None else bd.data_ptr(), y.ptr, ys.ptr if codes else 0, wp, wn, stream())
    torch.cuda.synchronize()
    return host(xd).reshape(N, S, C), y, ys


def check_norm(x, G, gamma, beta, x_type, y_type, kind, what, **kw):
    N, S, C = x.shape
    xr, y, ys = run_norm(x, G, gamma, beta, x_type, y_type, kind, **kw)
    ref, bound = O.group_norm(xr, G, gamma, beta, kw.get("eps", 1e-5), kind)
    if y_type != "e4m3":
        assert_close(host(y.rows()).reshape(N, S, C), ref, bound, y_type, what)
        y.check_guard()
        return
    ref, bound = ref.reshape(N * S, C), bound.reshape(N * S, C)
    code, scale = host(y.rows()).astype(np.float64), host(ys.rows()).astype(np.float64)
    for j in range(scale.shape[1]):
        part = slice(j * 128, (j + 1) * 128)
        a = np.maximum(np.abs(ref[:, part]).max(1), 2.0 ** -100)
        da = bound[:, part].max(1) + 4 * O.U * a
        assert np.all(np.abs(scale[:, j] * 448 - a) <= da), (what, j)
        t = ref[:, part] / scale[:, j:j + 1]
        c = code[:, part]
        # the nearest code of a value that may be off by its bound
        allowed = 0.5 * O.code_step(np.maximum(np.abs(t), np.abs(c))) + bound[:, part] / scale[:, j:j + 1] + 8 * O.U * np.abs(t)
        assert np.all(np.abs(c - t) <= allowed), (what, j)
        assert np.all(np.abs(c) <= 448)
    fill = -C % 16
    whole = y.raw.view(torch.uint8)[:N * S * y.row].view(N * S, y.row)
    assert int(whole[:, C:C + fill].max() if fill else 0) == 0
    y.check_guard(pad=fill)
    ys.check_guard()


@pytest.mark.parametrize("x_type,y_type", [(t, y) for t in ("f32", "f16", "bf16") for y in (t, "e4m3")])
@pytest.mark.parametrize("N,S,C,G,pad,lead", NORM_SHAPES)
def test_group_norm(N, S, C, G, pad, lead, x_type, y_type):
    x, gamma, beta = norm_inputs(N, S, C, N + S + C)
    kind = ("none", "relu", "silu")[(N + S + C + G) % 3]
    check_norm(x, G, gamma, beta, x_type, y_type, kind, (N, S, C, G, x_type, y_type, kind), pad=pad, lead=lead, y_pad=0 if pad == 0 else 5)


@pytest.mark.parametrize("x_type,y_type", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "e4m3"), ("f16", "e4m3"), ("bf16", "e4m3")])
@pytest.mark.parametrize("N,S,C,G,pad,lead", [(2, 30, 416, 32, 0, 0), (3, 40, 1152, 16, 0, 0), (2, 9, 1040, 16, 3, 1), (1, 400, 768, 16, 0, 0), (2, 100, 1152, 12, 8, 0),
                                              (1, 60, 156, 12, 0, 0), (1, 37, 1300, 100, 1, 0), (1, 200, 640, 2, 0, 0), (1, 2, 20000, 400, 0, 0)])
def test_group_norm_of_parts_of_samples(N, S, C, G, pad, lead, x_type, y_type):
    x, gamma, beta = norm_inputs(N, S, C, N + S + C)
    kind = ("none", "relu", "silu")[(N + S + C + G) % 3]
    check_norm(x, G, gamma, beta, x_type, y_type, kind, (N, S, C, G, x_type, y_type, kind), pad=pad, lead=lead, y_pad=0 if pad == 0 else 5)


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("with_gamma,with_beta", [(False, False), (True, False), (False, True)])
def test_group_norm_activations_and_missing_parameters(kind, with_gamma, with_beta):
    x, gamma, beta = norm_inputs(2, 100, 160, 9)
    for y_type in ("f32", "e4m3"):
        check_norm(x, 20, gamma if with_gamma else None, beta if with_beta else None, "f32", y_type, kind, (kind, with_gamma, with_beta, y_type))


def test_group_norm_of_far_off_means():
    """The mean a thousand times the spread: squares summed without it would lose everything."""
    rng = np.random.default_rng(3)
    for S in (50, 4000):
        x = 1000.0 + rng.normal(size=(2, S, 64))
        check_norm(x, 4, None, None, "f32", "f32", "none", S)


def test_group_norm_of_a_constant_is_beta():
    x = np.full((2, 30, 32), 3.25)
    beta = np.linspace(-1, 1, 32).astype(np.float32)
    for x_type in ("f32", "f16", "bf16"):
        _, y, _ = run_norm(x, 8, None, beta, x_type, x_type, "none")
        assert torch.equal(y.rows(), torch.from_numpy(beta).cuda().to(T[x_type]).expand(60, 32))


def test_group_norm_keeps_what_is_not_finite_in_its_group():
    x, gamma, beta = norm_inputs(2, 40, 64, 4)
    x[0, 7, 10] = np.nan                                      # sample 0, group 1 of 8
    x[1, 3, 63] = np.inf                                      # sample 1, group 7
    for S in (40,):
        _, y, _ = run_norm(x, 8, gamma, beta, "f32", "f32", "silu")
        nan = np.isnan(host(y.rows()).reshape(2, S, 8, 8))
        want = np.zeros_like(nan)
        want[0, :, 1] = want[1, :, 7] = True
        assert np.array_equal(nan, want)


@pytest.mark.parametrize("N,S,C,G", [(2, 49, 256, 32), (2, 3136, 64, 8)])
def test_group_norm_in_place_and_with_repeated_samples(N, S, C, G):
    x, gamma, beta = norm_inputs(N, S, C, 5)
    g, b = torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
    xd = torch.from_numpy(x).cuda().to(torch.float16)
    op = B.GroupNorm(N, S, C, G, x_type="f16", act="relu")
    ws, wp, wn = workspace(op)
    y = torch.empty_like(xd)
    op.forward(xd.data_ptr(), g.data_ptr(), b.data_ptr(), y.data_ptr(), 0, wp, wn, stream())
    z = xd.clone()
    op.forward(z.data_ptr(), g.data_ptr(), b.data_ptr(), z.data_ptr(), 0, wp, wn, stream())
    rep = B.GroupNorm(N, S, C, G, x_type="f16", act="relu", x_strides=(0, C))      # every sample is the first one
    w = torch.empty_like(xd)
    rep.forward(xd.data_ptr(), g.data_ptr(), b.data_ptr(), w.data_ptr(), 0, wp, wn, stream())
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    for n in range(N):
        assert torch.equal(w[n], y[0])


def test_group_norm_of_nothing():
    for N, S in ((0, 5), (5, 0)):
        op = B.GroupNorm(N, S, 32, 4)
        op.forward(0, 0, 0, 0, 0, 0, 0, stream())
    torch.cuda.synchronize()


# -- products ------------------------------------------------------------------------------------

def code_matrix(rng, M, K, rows, row, spread=1.0):
    """Codes [M, row] with NaN codes behind column K, their values and scales: quantised normal values."""
    code, scale = O.quantize((rng.normal(size=(M, K)) * spread * np.exp(0.5 * rng.normal(size=(M, 1)))).astype(np.float32), rows)
    raw = torch.full((M, row), NAN_CODE, dtype=torch.uint8)
    raw[:, :K] = torch.from_numpy(code).to(torch.float8_e4m3fn).view(torch.uint8)
    return raw, code, scale


def scale_table(scale, row):
    """Scales in rows `row` floats apart with NaN between them."""
    t = torch.full((scale.shape[0], row), float("nan"))
    t[:, :scale.shape[1]] = torch.from_numpy(scale)
    return t.cuda()


FORMS = ["rows", "64", "64 split", "128", "128 deep", "256"]


def product_form(M, N, kbytes, E=0, widest=True):
    """The form that a product runs in: the estimate of csrc/op_matmul.hip."""
    cd = lambda a, b: -(-a // b)  # noqa: E731
    slabs, w = cd(kbytes, 128), (cd(M, 16) + min(E, M)) * cd(N, 16)
    if w <= 512 or (not E and M <= 16):
        return "rows"
    best = None
    for form, size, places, start, slab, half in (("64", 64, 512, 1.5, 0.41, 0.20), ("64 split", 64, 256, 2.3, 0.24, 0.16), ("128", 128, 512, 3.6, 0.88, 0.67),
                                                  ("128 deep", 128, 256, 2.2, 0.62, 0.50), ("256", 256, 256, 6.2, 1.38, 1.25)):
        if form == "256" and not widest:
            continue
        full, rest = divmod(int(np.ceil(cd(M, size) + 0.5 * E)) * cd(N, size), places)
        t = max(7.2, 3.0 + slabs * (full * slab + (0 if rest == 0 else half if rest <= places / 2 else slab)) + (full + (rest > 0)) * start)
        if best is None or t < best[0]:
            best = (t, form)
    return best[1]


MATMUL_SHAPES = [  # M, N, K
    (1, 1, 1), (1, 16, 128), (1, 100, 300), (1, 512, 4096), (1, 2049, 640), (2, 64, 1000), (3, 130, 17), (8, 1024, 512), (15, 200, 129), (16, 256, 2048),
    (17, 257, 256), (32, 96, 1100), (33, 512, 384), (64, 64, 64), (65, 130, 100), (100, 1000, 260), (127, 128, 128), (129, 300, 300),
    (200, 2048, 512), (256, 256, 256), (257, 511, 640), (333, 1000, 1100), (700, 70, 900), (1000, 1030, 129), (2100, 520, 272),
    (4100, 4100, 272), (300, 700, 3000), (1500, 900, 1300), (2000, 1100, 1000),
]


@pytest.mark.parametrize("y_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,N,K", MATMUL_SHAPES)
def test_matmul_blocks(M, N, K, y_type):
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    kind = ("none", "relu", "silu")[(M + N + K) % 3]
    odd = (M + N) % 2                                          # wider rows, y not on 16 bytes
    kb, row = -(-K // 128), -(-K // 16) * 16 + 16 * odd
    ra, ca, sa = code_matrix(rng, M, K, 1, row)
    rb, cb, sb = code_matrix(rng, N, K, 128, row, 0.05)
    a, b = ra.cuda(), rb.cuda()
    asc, bsc = scale_table(sa, kb + odd), scale_table(sb, kb + 2 * odd)
    bias = (0.2 * rng.normal(size=N)).astype(np.float32) if (M + K) % 2 else None
    bd = None if bias is None else torch.from_numpy(bias).cuda()
    y = Out(M, N, y_type, N + 3 * odd, odd)
    op = B.BlockMatmul(M, N, K, y_type=T[y_type], act=kind, a_row=row, b_row=row, y_row=N + 3 * odd, a_scale_row=kb + odd, b_scale_row=kb + 2 * odd)
    ws, wp, wn = workspace(op)
    op.forward(a.data_ptr(), asc.data_ptr(), b.data_ptr(), bsc.data_ptr(), 0 if bd is None else bd.data_ptr(), y.ptr, wp, wn, stream())
    torch.cuda.synchronize()
    ref, bound = O.product(O.values(ca, sa, 1), O.values(cb, sb, 128), bias, kind, cores8=y_type != "f32")
    assert_close(host(y.rows()), ref, bound, y_type, (M, N, K, kind))
    y.check_guard()


@pytest.mark.parametrize("y_type", ["f16", "bf16"])
def test_matmul_blocks_on_the_widest_tile(y_type):
    """Rows picked all over the matrix against the definition; the sizes are not multiples of anything."""
    M, N, K = 4090, 4090, 1100
    assert product_form(M, N, K) == "256"
    rng = np.random.default_rng(5)
    kb, row = -(-K // 128), -(-K // 16) * 16
    ra, ca, sa = code_matrix(rng, M, K, 1, row)
    rb, cb, sb = code_matrix(rng, N, K, 128, row, 0.05)
    bias = (0.2 * rng.normal(size=N)).astype(np.float32)
    a, b, asc, bsc, bd = ra.cuda(), rb.cuda(), scale_table(sa, kb), scale_table(sb, kb), torch.from_numpy(bias).cuda()
    y = Out(M, N, y_type)
    op = B.BlockMatmul(M, N, K, y_type=T[y_type], act="silu", a_row=row, b_row=row)
    ws, wp, wn = workspace(op)
    op.forward(a.data_ptr(), asc.data_ptr(), b.data_ptr(), bsc.data_ptr(), bd.data_ptr(), y.ptr, wp, wn, stream())
    torch.cuda.synchronize()
    at = sorted(set(range(0, M, 41)) | set(range(250, 262)) | set(range(M - 5, M)))
    ref, bound = O.product(O.values(ca[at], sa[at], 1), O.values(cb, sb, 128), bias, "silu", cores8=True)
    assert_close(host(y.rows()[at]), ref, bound, y_type, (M, N, K))
    y.check_guard()


def test_every_form_of_the_products_is_looked_at():
    """The shapes of the tests reach every form in every type (32-bit results of codes have no widest tile)."""
    whole = {product_form(M, N, K) for M, N, K in MATMUL_SHAPES} | {"256"}
    assert whole == set(FORMS)
    assert {product_form(M, N, K, widest=False) for M, N, K in MATMUL_SHAPES} == set(FORMS[:-1])


def test_matmul_blocks_twice_gives_the_same_bits():
    rng = np.random.default_rng(1)
    for M, N, K in ((1, 512, 8192), (40, 256, 8192), (500, 300, 700)):
        kb, row = -(-K // 128), -(-K // 16) * 16
        ra, _, sa = code_matrix(rng, M, K, 1, row)
        rb, _, sb = code_matrix(rng, N, K, 128, row)
        a, b, asc, bsc = ra.cuda(), rb.cuda(), scale_table(sa, kb), scale_table(sb, kb)
        op = B.BlockMatmul(M, N, K, y_type="f32")
        ws, wp, wn = workspace(op)
        got = []
        for _ in range(3):
            y = torch.empty(M, N, device="cuda")
            op.forward(a.data_ptr(), asc.data_ptr(), b.data_ptr(), bsc.data_ptr(), 0, y.data_ptr(), wp, wn, stream())
            got.append(y)
        torch.cuda.synchronize()
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_matmul_blocks_keeps_what_is_not_finite_in_its_row_and_column():
    rng = np.random.default_rng(2)
    for M in (3, 40, 300):
        N, K = 200, 384
        ra, ca, sa = code_matrix(rng, M, K, 1, K)
        rb, cb, sb = code_matrix(rng, N, K, 128, K)
        ra[1, 200] = NAN_CODE
        rb[130, 5] = NAN_CODE
        sa[2, 1] = np.inf
        a, b, asc, bsc = ra.cuda(), rb.cuda(), scale_table(sa, 3), scale_table(sb, 3)
        y = Out(M, N, "f32")
        op = B.BlockMatmul(M, N, K, y_type="f32")
        ws, wp, wn = workspace(op)
        op.forward(a.data_ptr(), asc.data_ptr(), b.data_ptr(), bsc.data_ptr(), 0, y.ptr, wp, wn, stream())
        torch.cuda.synchronize()
        got = host(y.rows())
        bad = np.zeros((M, N), bool)
        bad[1] = bad[2] = True
        bad[:, 130] = True
        assert np.all(np.isfinite(got[~bad])), M
        assert np.all(np.isnan(got[1])) and np.all(np.isnan(got[:, 130])) and not np.any(np.isfinite(got[2])), M


def test_matmul_blocks_of_no_rows():
    B.BlockMatmul(0, 16, 16).forward(0, 0, 0, 0, 0, 0, 0, 0, stream())
    torch.cuda.synchronize()


# -- products grouped by expert --------------------------------------------------------------------

GROUPS = {  # what each expert gets
    "even": [40, 40, 40, 40], "ragged": [0, 1, 130, 0, 17, 64, 3], "one": [0, 0, 200, 0], "single rows": [1] * 9 + [0] * 7,
    "last": [0, 0, 0, 77], "large": [300, 513, 2], "few": [0, 2, 0, 1, 5], "many": [(7 * e) % 11 for e in range(70)],
    "thousands": [1500, 0, 2700, 3999],
}


def run_grouped(rng, counts, N, K, a_type, y_type, kind, gather, bias, odd, first=0, beyond=0, some=1):
    """One call with `first` rows before the first group and `beyond` behind the last (some: see below); the rows that the groups cover, what came
    out, the exact result and its bound."""
    E, T_ = len(counts), sum(counts)
    M = first + T_ + beyond
    offsets = np.cumsum([first] + list(counts)).astype(np.int32)
    have = max(3, M // 2) if gather else M
    index = rng.integers(0, have, size=M).astype(np.int32) if gather else None
    if gather and M > 2:
        index[first + 1] = -1                                 # stand for rows of zeros
        index[M - 1] = have
    codes = a_type == "e4m3"
    unit = 16 if codes else 8
    row, kb, nb = -(-K // unit) * unit + unit * odd, -(-K // 128), -(-N // 128)
    if codes:
        ra, ca, sa = code_matrix(rng, have, K, 1, row)
        parts = [code_matrix(rng, N, K, 128, row, 0.05) for _ in range(E)]
        a, b = ra.cuda(), torch.stack([p[0] for p in parts]).cuda()
        asc = scale_table(sa, kb + odd)
        bsc = torch.stack([scale_table(p[2], kb) for p in parts])
        av = O.values(ca, sa, 1)
        bv = [O.values(p[1], p[2], 128) for p in parts]
    else:
        abuf, a = rows_of(rng.normal(size=(have, K)), a_type, row)
        bbuf, b = rows_of(rng.normal(size=(E * N, K)) * K ** -0.5, a_type, row)
        asc = bsc = None
        av, bv = host(a).astype(np.float64), list(host(b).astype(np.float64).reshape(E, N, K))
    bias_h = (0.2 * rng.normal(size=(E, N))).astype(np.float32) if bias else None
    bd = None if bias_h is None else torch.from_numpy(bias_h).cuda()
    off, idx = torch.from_numpy(offsets).cuda(), None if index is None else torch.from_numpy(index).cuda()
    y = Out(M, N, y_type, N + 3 * odd, odd)
    op = B.GroupedMatmul(M, N, K, E, a_type=T[a_type], y_type=T[y_type], act=kind, a_rows=have, a_row=row, b_row=row, y_row=N + 3 * odd,
                         a_scale_row=kb + odd if codes else 0, b_scale_row=kb if codes else 0, b_scale_expert=nb * kb if codes else 0)
    ws, wp, wn = workspace(op)
    ptr = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    op.forward(a.data_ptr(), ptr(asc), ptr(idx), off.data_ptr(), b.data_ptr(), ptr(bsc), ptr(bd), y.ptr, wp, wn, stream())
    torch.cuda.synchronize()
    if index is not None:
        av = np.concatenate([av, np.zeros((1, K))])[np.where((index < 0) | (index >= have), have, index)]
    ref, bound = np.zeros((M, N)), np.zeros((M, N))
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        if hi > lo:                                           # (some > 1: each some-th row and the ends)
            at = sorted(set(range(lo, hi, some)) | {lo, hi - 1})
            ref[at], bound[at] = O.product(av[at], bv[e], None if bias_h is None else bias_h[e], kind, blocks=codes, cores8=codes and y_type != "f32")
    return range(first, first + T_), y, ref, bound


@pytest.mark.parametrize("a_type,y_type", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32"), ("e4m3", "bf16"), ("e4m3", "f32"), ("e4m3", "f16")])
@pytest.mark.parametrize("groups", list(GROUPS))
def test_matmul_grouped(groups, a_type, y_type):
    counts = GROUPS[groups]
    rng = np.random.default_rng(len(groups) * 31 + sum(counts))
    for i, (N, K) in enumerate(((64, 128), (130, 200), (257, 520), (1, 1), (512, 1024)) if groups != "thousands" else ((2060, 200), (2048, 128), (300, 1200))):
        if groups == "many" and K > 600:
            continue
        gather, bias, odd = (i + len(counts)) % 2 == 1, i % 3 == 1, i % 2
        kind = ("none", "relu", "silu")[i % 3]
        print("case", groups, a_type, y_type, N, K, gather, bias, kind, flush=True)
        covered, y, ref, bound = run_grouped(rng, counts, N, K, a_type, y_type, kind, gather, bias, odd, first=5 * (i == 2), beyond=9 * (i == 2))
        got = host(y.rows())
        assert_close(got[covered.start:covered.stop], ref[covered.start:covered.stop], bound[covered.start:covered.stop], y_type, (groups, N, K, kind))
        y.check_guard(covered)


@pytest.mark.parametrize("a_type,y_type", [("f16", "f16"), ("bf16", "f32"), ("e4m3", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("form", FORMS[1:])
def test_matmul_grouped_in_every_form(form, a_type, y_type):
    """Unequal groups in each of the tiles, rows picked by an index, some of which stand for zeros; every 17th row and the ends of the
    groups against the definition."""
    codes = a_type == "e4m3"
    # (columns, summed bytes, rows of the groups)
    N, kbytes, counts = {"64": (700, 400, [300, 0, 900, 401]), "64 split": (330, 3300, [200, 0, 300, 101]), "128": (2060, 400, [1500, 0, 2700, 3999]),
                         "128 deep": (1000, 2500, [700, 0, 1000, 901]), "256": (4090, 2400, [900, 0, 1200, 1197])}[form]
    if form == "256" and codes and y_type == "f32":
        return
    K = kbytes // (1 if codes else 2)
    assert product_form(sum(counts), N, kbytes, len(counts), not (codes and y_type == "f32")) == form
    rng = np.random.default_rng(len(form))
    covered, y, ref, bound = run_grouped(rng, counts, N, K, a_type, y_type, "silu", True, True, 0, some=17)
    at = ref.any(1) | bound.any(1)
    assert at.sum() > sum(counts) // 17
    got = host(y.rows())
    assert_close(got[at], ref[at], bound[at], y_type, (form, a_type, y_type))
    y.check_guard(covered)


def test_matmul_grouped_with_offsets_that_are_out_of_range():
    """Offsets are clamped into the rows that there are: nothing outside is read or written."""
    E, N, K, M = 4, 96, 64, 50
    a = torch.randn(M, K, device="cuda", dtype=torch.float16)
    b = torch.randn(E, N, K, device="cuda", dtype=torch.float16)
    op = B.GroupedMatmul(M, N, K, E, a_type="f16")
    ws, wp, wn = workspace(op)
    for off, ok in (([-7, 10, 10, 30, 1000], range(0, 50)), ([60, 70, 80, 90, 100], range(0, 0)), ([-9, -8, -7, -6, -5], range(0, 0))):
        y = Out(M, N, "f16")
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        op.forward(a.data_ptr(), 0, 0, o.data_ptr(), b.data_ptr(), 0, 0, y.ptr, wp, wn, stream())
        torch.cuda.synchronize()
        y.check_guard(ok)
        clamped = [min(max(v, 0), M) for v in off]
        for e in range(E):
            lo, hi = clamped[e], clamped[e + 1]
            if hi > lo:
                ref = a[lo:hi].float() @ b[e].float().t()
                assert torch.allclose(y.rows()[lo:hi].float(), ref, rtol=2e-3, atol=2e-2)


def test_matmul_grouped_of_no_rows():
    B.GroupedMatmul(0, 16, 16, 2, a_type="f16").forward(0, 0, 0, 0, 0, 0, 0, 0, 0, 0, stream())
    torch.cuda.synchronize()


# -- how they are called ---------------------------------------------------------------------------

def test_torch_conveniences_and_the_example():
    """The block of examples/channels_last_experts.py: norm to codes, router, grouped products, against the same in 32 bits.  Codes are off
    by up to 2^-4 of a value (3 % rms), and two products follow one another: a few percent of what the block adds."""
    import importlib.util
    import os
    spec = importlib.util.spec_from_file_location("example", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "channels_last_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(2, 7, 9, 192) < 0.1
    assert m.main(1, 1, 1, 64) < 0.1


def test_torch_conveniences_refuse():
    x = torch.zeros(2, 4, 32, device="cuda", dtype=torch.float16)
    with pytest.raises(ValueError):
        B.group_norm_torch(x.transpose(1, 2), 4)
    with pytest.raises(ValueError):
        B.group_norm_torch(x, 4, gamma=torch.ones(32, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        B.quantize_blocks_torch(torch.zeros(4, 32))
    q, s = B.quantize_blocks_torch(torch.zeros(4, 32, device="cuda"))
    w, t = B.quantize_blocks_torch(torch.zeros(4, 48, device="cuda"), 128)
    with pytest.raises(ValueError):
        B.matmul_blocks_torch(q, s, w, t)
    with pytest.raises(ValueError):
        B.matmul_grouped_torch(x[0], x.bfloat16(), torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        B.matmul_grouped_torch(x[0], x, torch.zeros(3, dtype=torch.int64, device="cuda"))


def _calls():
    """One call of each operator (of each form of the group norm and the products) on its own buffers: (run, outputs)."""
    rng = np.random.default_rng(11)
    out = []
    for N, S, C, G, y_type in ((2, 49, 256, 32, "f16"), (2, 3000, 48, 3, "f16"), (1, 500, 360, 30, "e4m3")):
        x, gamma, beta = norm_inputs(N, S, C, 6)
        xd, g, b = torch.from_numpy(x).cuda().half(), torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda()
        y = B.empty_codes(N * S, C) if y_type == "e4m3" else torch.empty_like(xd)
        ys = torch.empty(N * S, -(-C // 128), device="cuda")
        op = B.GroupNorm(N, S, C, G, act="silu", x_type="f16", y_type=y_type)
        ws, wp, wn = workspace(op)
        keep = (xd, g, b, ws)
        out.append((lambda st, op=op, y=y, ys=ys, wp=wp, wn=wn, k=keep: op.forward(k[0].data_ptr(), k[1].data_ptr(), k[2].data_ptr(), y.data_ptr(), ys.data_ptr(), wp, wn, st), y, xd))
    x = torch.from_numpy(rng.normal(size=(200, 300)).astype(np.float32)).cuda()
    for rows in (1, 128):
        q, s = B.empty_codes(200, 300), torch.empty(-(-200 // rows), 3, device="cuda")
        op = B.BlockQuantizer(200, 300, rows=rows, x_type="f32")
        out.append((lambda st, op=op, q=q, s=s: op.forward(x.data_ptr(), q.data_ptr(), s.data_ptr(), st), q, x))
    for M, N, K in ((3, 200, 600), (100, 600, 300), (1000, 2100, 300)):
        a, sa = B.quantize_blocks_torch(torch.from_numpy(rng.normal(size=(M, K)).astype(np.float32)).cuda())
        b, sb = B.quantize_blocks_torch(torch.from_numpy(rng.normal(size=(N, K)).astype(np.float32)).cuda(), 128)
        y = torch.empty(M, N, device="cuda")
        op = B.BlockMatmul(M, N, K, y_type="f32")
        ws, wp, wn = workspace(op)
        out.append((lambda st, op=op, y=y, k=(a, sa, b, sb, ws), wp=wp, wn=wn: op.forward(k[0].data_ptr(), k[1].data_ptr(), k[2].data_ptr(), k[3].data_ptr(), 0, y.data_ptr(), wp, wn, st), y, sa))
    for counts in ([3, 0, 5], [100, 300, 2]):
        off = torch.tensor(np.cumsum([0] + counts), dtype=torch.int32, device="cuda")
        a, b = torch.randn(sum(counts), 256, device="cuda").half(), torch.randn(3, 1100, 256, device="cuda").half()
        y = torch.empty(sum(counts), 1100, device="cuda", dtype=torch.float16)
        op = B.GroupedMatmul(sum(counts), 1100, 256, 3, a_type="f16")
        ws, wp, wn = workspace(op)
        out.append((lambda st, op=op, y=y, k=(a, b, off, ws), wp=wp, wn=wn: op.forward(k[0].data_ptr(), 0, 0, k[2].data_ptr(), k[1].data_ptr(), 0, 0, y.data_ptr(), wp, wn, st), y, a))
    return out


def test_operators_on_another_stream_and_in_a_graph():
    """Every call on a stream of its own after an input changed on it, then captured and replayed, inputs changing between the replays."""
    s = torch.cuda.Stream()
    for i, (run, y, x) in enumerate(_calls()):
        print("case", i, tuple(y.shape), y.dtype, flush=True)
        results = []
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for k in range(3):
                x.mul_(2.0 if k == 1 else 1.0)
                y.view(torch.uint8).zero_()
                run(s.cuda_stream)
                results.append(y.clone())
        s.synchronize()
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
            assert torch.equal(y.view(torch.uint8), results[k].view(torch.uint8)), (i, k)
            torch.zeros(1000, device="cuda").sum().item()         # other work between the replays


def test_rows_further_than_32_bits_reach():
    """Activations and results whose last rows lie beyond 2^32 bytes."""
    M, N, K, row = 1100, 96, 128, 1 << 22
    a = torch.zeros(M, row - 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)      # 4.6 GB
    q, s = B.quantize_blocks_torch(torch.randn(M, K, device="cuda"))
    a[:, :K] = q
    b, t = B.quantize_blocks_torch(torch.randn(N, K, device="cuda"), 128)
    want = B.matmul_blocks_torch(q, s, b, t, dtype=torch.float32)
    got = B.matmul_blocks_torch(a[:, :K], s, b, t, dtype=torch.float32)
    assert torch.equal(got, want)
    idx = torch.arange(M - 1, -1, -1, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    flipped = B.matmul_grouped_torch(a[:, :K], b[None], off, s, t[None], index=idx, dtype=torch.float32)
    assert torch.equal(flipped, want.flip(0))


def test_torch_conveniences_refuse_scales_and_integers_that_do_not_fit():
    q, s = B.quantize_blocks_torch(torch.randn(8, 300, device="cuda"))
    w, t = B.quantize_blocks_torch(torch.randn(2, 200, 300, device="cuda"), 128)
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    assert s.shape == (8, 3) and t.shape == (2, 2, 3)
    for bad in (s[:, :2], s[:7], s.double(), s.cpu(), s.t().contiguous().t(), None):
        with pytest.raises(ValueError):
            B.matmul_blocks_torch(q, bad, w[0], t[0])
        with pytest.raises(ValueError):
            B.matmul_grouped_torch(q, w, off, bad, t)
    for bad in (t[:, :1], t[:1], t.half(), None):
        with pytest.raises(ValueError):
            B.matmul_grouped_torch(q, w, off, s, bad)
    with pytest.raises(ValueError):
        B.matmul_blocks_torch(q.float().half(), s, w[0].float().half(), t[0])
    for bad in (off.cpu(), off.long(), off[:2], torch.stack([off, off], 1)[:, 0]):
        with pytest.raises(ValueError):
            B.matmul_grouped_torch(q, w, bad, s, t)
    for bad in (off.cpu(), off.long(), torch.stack([off, off], 1)[:, 0]):
        with pytest.raises(ValueError):
            B.matmul_grouped_torch(q, w, off, s, t, index=bad)
    assert B.matmul_grouped_torch(q, w, off, s, t, index=off[:2]).shape == (2, 200)
