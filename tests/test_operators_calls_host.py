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
