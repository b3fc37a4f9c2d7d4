"""The torch conveniences of the operators without a GPU: tensors that have a device, types and strides but no memory, and calls that are
noted instead of made."""
import contextlib
import warnings

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2112_15445_amd import binding as B


@pytest.fixture
def calls(monkeypatch):
    """[(operator, arguments, current device)] of the calls made, with cuda:0 current at the start; streams are numbered 100 + device."""
    made, current = [], [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d).index if not isinstance(d, int) else d
        try:
            yield
        finally:
            current[0] = before

    class Stream:
        def __init__(self, d):
            self.cuda_stream = 100 + (current[0] if d is None else torch.device(d).index)

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(d))
    for op in (B.GroupNorm, B.BlockQuantizer, B.BlockMatmul, B.GroupedMatmul):
        monkeypatch.setattr(op, "forward", lambda self, *a: made.append((self, a, current[0])))
    with FakeTensorMode(), warnings.catch_warnings():
        warnings.simplefilter("ignore")              # (these tensors' address is 0)
        yield made


def tensor(*shape, dtype=torch.float16, device="cuda:0"):
    return torch.empty(*shape, dtype=dtype, device=device)


def codes(*shape, device="cuda:0"):
    return B.empty_codes(*shape, device=device)


@pytest.mark.parametrize("default", [torch.float16, torch.bfloat16, torch.float64])
def test_scales_are_32_bit_floats_whatever_the_default_type(calls, default):
    was = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        scales = [B.group_norm_torch(tensor(2, 5, 320), 8, codes=True)[1], B.quantize_blocks_torch(tensor(9, 300))[1], B.quantize_blocks_torch(tensor(3, 200, 300), 128)[1]]
    finally:
        torch.set_default_dtype(was)
    assert [s.dtype for s in scales] == [torch.float32] * 3
    assert [tuple(s.shape) for s in scales] == [(10, 3), (9, 3), (3, 2, 3)]
    assert len(calls) == 5


def test_a_stack_of_weights_is_no_matrix(calls):
    """Square experts [E, K, K] with the scales that belong to them look like E columns of K values."""
    a, s = codes(6, 256), tensor(6, 2, dtype=torch.float32)
    for E, N in ((4, 256), (2, 256), (256, 256)):
        with pytest.raises(ValueError):
            B.matmul_blocks_torch(a, s, codes(E, N, 256), tensor(E, 2, 2, dtype=torch.float32))
    with pytest.raises(ValueError):
        B.matmul_blocks_torch(codes(2, 6, 256), tensor(2, 6, 2, dtype=torch.float32), codes(256, 256), tensor(2, 2, dtype=torch.float32))
    assert not calls
    assert B.matmul_blocks_torch(a, s, codes(40, 256), tensor(1, 2, dtype=torch.float32)).shape == (6, 40)


def test_calls_are_made_on_the_device_of_the_tensors(calls):
    """cuda:0 is current and the tensors lie on cuda:1: the call is made with cuda:1 current and on its stream, and cuda:0 is current again."""
    on = "cuda:1"
    q, s = B.group_norm_torch(tensor(2, 5, 256, device=on), 8, tensor(256, dtype=torch.float32, device=on), tensor(256, dtype=torch.float32, device=on), codes=True)
    B.group_norm_torch(tensor(1, 3000, 48, device=on), 3)                      # (takes a workspace)
    w, t = B.quantize_blocks_torch(tensor(2, 200, 256, device=on), 128)
    B.matmul_blocks_torch(q, s, w[0], t[0], bias=tensor(200, dtype=torch.float32, device=on))
    B.matmul_grouped_torch(q, w, tensor(3, dtype=torch.int32, device=on), s, t)
    assert [c[2] for c in calls] == [1] * 6 and [c[1][-1] for c in calls] == [101] * 6
    assert q.device == s.device == w.device == t.device == torch.device(on)
    assert torch.cuda.current_stream().cuda_stream == 100


def test_convolutions_are_made_on_the_device_of_the_tensors(calls):
    class Plan:
        dtype = B.SC_F32

        class layer:
            D = 4

        def info(self):
            class I:
                P = Q = 3
            return I

        def workspace_size(self, n):
            return 64

        def forward(self, *a):
            calls.append((self, a, torch.cuda.current_stream().cuda_stream - 100))

    y = B.forward_torch(Plan(), tensor(2, 3, 5, 5, dtype=torch.float32, device="cuda:1"))
    assert y.device == torch.device("cuda:1") and calls[0][2] == 1 and calls[0][1][-1] == 101


def test_parameters_on_another_device_are_refused(calls):
    there = tensor(64, dtype=torch.float32, device="cuda:1")
    for pair in ((there, None), (None, there)):
        with pytest.raises(ValueError):
            B.group_norm_torch(tensor(2, 5, 64), 8, *pair)
    with pytest.raises(ValueError):
        B.matmul_blocks_torch(codes(3, 128), tensor(3, 1, dtype=torch.float32), codes(64, 128), tensor(1, 1, dtype=torch.float32), bias=there)
    with pytest.raises(ValueError):
        B.matmul_grouped_torch(tensor(3, 128), tensor(2, 32, 128), tensor(3, dtype=torch.int32), bias=there)
    assert not calls


def test_tensors_that_want_a_gradient_are_refused(calls):
    """The operators are forward only: a result without a gradient would end it silently.  Under no_grad nobody expects one."""
    f32 = dict(dtype=torch.float32)
    with_grad = lambda t: t.requires_grad_()  # noqa: E731
    off = tensor(3, dtype=torch.int32)
    a, b, sa, sb = codes(6, 256), codes(2, 64, 256), tensor(6, 2, **f32), tensor(2, 1, 2, **f32)
    wanting = [
        lambda: B.group_norm_torch(with_grad(tensor(2, 5, 64)), 8),
        lambda: B.group_norm_torch(tensor(2, 5, 64), 8, gamma=with_grad(tensor(64, **f32))),
        lambda: B.group_norm_torch(tensor(2, 5, 64), 8, beta=with_grad(tensor(64, **f32)), codes=True),
        lambda: B.quantize_blocks_torch(with_grad(tensor(5, 64)), 128),
        lambda: B.matmul_blocks_torch(a, with_grad(tensor(6, 2, **f32)), b[0], sb[0]),
        lambda: B.matmul_blocks_torch(a, sa, b[0], with_grad(tensor(1, 2, **f32))),
        lambda: B.matmul_blocks_torch(a, sa, b[0], sb[0], bias=with_grad(tensor(64, **f32))),
        lambda: B.matmul_grouped_torch(with_grad(tensor(6, 128)), tensor(2, 64, 128), off),
        lambda: B.matmul_grouped_torch(tensor(6, 128), with_grad(tensor(2, 64, 128)), off),
        lambda: B.matmul_grouped_torch(a, b, off, with_grad(tensor(6, 2, **f32)), sb),
        lambda: B.matmul_grouped_torch(a, b, off, sa, with_grad(tensor(2, 1, 2, **f32))),
        lambda: B.matmul_grouped_torch(a, b, off, sa, sb, bias=with_grad(tensor(2, 64, **f32))),
    ]
    for i, call in enumerate(wanting):
        with pytest.raises(ValueError, match="gradient"):
            call()
        assert not calls, i
    with torch.no_grad():
        for call in wanting:
            call()
    assert len(calls) == len(wanting)
