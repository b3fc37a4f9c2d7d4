"""The torch conveniences around a layer of experts without a GPU: tensors that have a device, types and strides but no memory, and calls that are noted
instead of made."""
import contextlib
import warnings

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2112_15445_amd import binding as B

F32, I32 = dict(dtype=torch.float32), dict(dtype=torch.int32)


@pytest.fixture
def calls(monkeypatch):
    """[(operator, arguments, current device, backward)] of the calls made, with cuda:0 current at the start; streams are numbered 100 + device."""
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
    for op in (B.ExpertRouter, B.ExpertSort, B.RowGather, B.RowCombine, B.Adapters):
        monkeypatch.setattr(op, "forward", lambda self, *a: made.append((self, a, current[0], False)))
        if hasattr(op, "backward"):
            monkeypatch.setattr(op, "backward", lambda self, *a: made.append((self, a, current[0], True)))
    with FakeTensorMode(), warnings.catch_warnings():
        warnings.simplefilter("ignore")              # (these tensors' address is 0)
        yield made


def tensor(*shape, dtype=torch.float16, device="cuda:0"):
    return torch.empty(*shape, dtype=dtype, device=device)


def one_of_each(on="cuda:0", change=lambda name, t: t):
    """{call: what it returns}, each tensor argument through change(its name, it)."""
    def t(name, *shape, **kw):
        return change(name, tensor(*shape, device=on, **kw))

    return {
        "route": lambda: B.route_experts_torch(t("logits", 6, 40), 3, bias=t("bias", 40, **F32)),
        "route back": lambda: B.route_experts_backward_torch(t("logits", 6, 40), t("ids", 6, 3, **I32), t("dweights", 6, 3, **F32)),
        "sort": lambda: B.sort_by_expert_torch(t("ids", 6, 3, **I32), 40),
        "gather": lambda: B.gather_rows_torch(t("x", 6, 64), t("index", 9, **I32)),
        "combine": lambda: B.combine_rows_torch(t("x", 18, 64), t("position", 6, 3, **I32), t("weights", 6, 3, **F32), t("residual", 6, 64)),
        "combine back": lambda: B.combine_rows_backward_torch(t("dy", 6, 64), t("x", 18, 64), t("position", 6, 3, **I32), t("weights", 6, 3, **F32)),
        "adapters": lambda: B.adapters_torch(t("y", 6, 64, **F32), t("x", 6, 128), t("a", 2, 8, 128), t("b", 2, 64, 8), t("offsets", 3, **I32), t("index", 6, **I32), t("scale", 2, **F32)),
    }


def test_calls_are_made_on_the_device_of_the_tensors(calls):
    for name, call in one_of_each("cuda:1").items():
        out = call()
        op, args, device, back = calls[-1]
        assert device == 1 and args[-1] == 101 and back == name.endswith("back"), name
        assert all(v.device == torch.device("cuda:1") for v in (out if isinstance(out, tuple) else (out,)))
    assert len(calls) == 7


def test_what_they_return(calls):
    each = one_of_each()
    ids, w = each["route"]()
    assert (tuple(ids.shape), ids.dtype, tuple(w.shape), w.dtype) == ((6, 3), torch.int32, (6, 3), torch.float32)
    assert tuple(each["route back"]().shape) == (6, 40)
    off, index, position = each["sort"]()
    assert (tuple(off.shape), tuple(index.shape), tuple(position.shape)) == ((41,), (18,), (6, 3))
    assert tuple(B.sort_by_expert_torch(tensor(6, **I32), 4)[2].shape) == (6,)
    assert tuple(each["gather"]().shape) == (9, 64) and tuple(each["combine"]().shape) == (6, 64)
    dx, dw = each["combine back"]()
    assert tuple(dx.shape) == (18, 64) and tuple(dw.shape) == (6, 3)
    assert each["adapters"]().dtype == torch.float32
    codes = B.gather_rows_torch(B.empty_codes(6, 100, device="cuda:0"), tensor(9, **I32))
    assert codes.dtype == torch.float8_e4m3fn and codes.stride(0) == 112


@pytest.mark.parametrize("wrong", ["device", "type", "strides"])
def test_tensors_that_do_not_fit_are_refused(calls, wrong):
    """Each argument in its turn on another device, of another type, or with columns apart."""
    seen = []
    for name, call in one_of_each(change=lambda n, t: seen.append(n) or t).items():
        del seen[:]
        call()
        for arg in list(seen):
            # the first tensor says where the call is made, and of what type
            if wrong == "device" and (arg == seen[0] or arg == "dy") and name != "combine back" or wrong == "type" and arg in ("logits", "x", "dy") or wrong == "strides" and arg == "y":
                continue

            def change(n, t, arg=arg):
                if n != arg:
                    return t
                if wrong == "device":
                    return torch.empty_like(t, device="cuda:1")
                if wrong == "type":
                    return t.to({torch.float32: torch.float64, torch.int32: torch.int64, torch.float16: torch.float32}[t.dtype])
                return torch.empty(*t.shape, 2, dtype=t.dtype, device=t.device)[..., 0]

            before = len(calls)
            if name == "adapters" and wrong == "type" and arg == "y":
                continue
            with pytest.raises((ValueError, KeyError)):
                one_of_each(change=change)[name]()
            assert len(calls) == before, (name, arg)
        del calls[:]


def test_tensors_that_want_a_gradient_are_refused(calls):
    for arg in ("logits", "bias", "dweights", "x", "weights", "residual", "dy", "y", "a", "b", "scale"):
        for name, call in one_of_each(change=lambda n, t: t.requires_grad_() if n == arg else t).items():
            if arg not in {"route": ("logits", "bias"), "route back": ("logits", "dweights"), "sort": (), "gather": ("x",), "combine": ("x", "weights", "residual"),
                           "combine back": ("dy", "x", "weights"), "adapters": ("y", "x", "a", "b", "scale")}[name]:
                continue
            before = len(calls)
            with pytest.raises(ValueError, match="gradient"):
                call()
            assert len(calls) == before
            with torch.no_grad():
                call()


def test_shapes_that_do_not_belong_together_are_refused(calls):
    bad = [
        lambda: B.route_experts_torch(tensor(2, 6, 40), 3),
        lambda: B.route_experts_torch(tensor(6, 40), 3, bias=tensor(39, **F32)),
        lambda: B.route_experts_backward_torch(tensor(6, 40), tensor(6, 3, **I32), tensor(6, 2, **F32)),
        lambda: B.sort_by_expert_torch(tensor(6, 3, 2, **I32), 4),
        lambda: B.gather_rows_torch(tensor(2, 6, 64), tensor(9, **I32)),
        lambda: B.gather_rows_torch(tensor(6, 64), tensor(3, 3, **I32)),
        lambda: B.combine_rows_torch(tensor(18, 64), tensor(18, **I32)),
        lambda: B.combine_rows_torch(tensor(18, 64), tensor(6, 3, **I32), tensor(6, 2, **F32)),
        lambda: B.combine_rows_torch(tensor(18, 64), tensor(6, 3, **I32), residual=tensor(6, 32)),
        lambda: B.combine_rows_torch(tensor(18, 64), tensor(6, 3, **I32), residual=tensor(6, 64, **F32)),
        lambda: B.combine_rows_backward_torch(tensor(5, 64), tensor(18, 64), tensor(6, 3, **I32)),
        lambda: B.adapters_torch(tensor(6, 64), tensor(5, 128), tensor(2, 8, 128), tensor(2, 64, 8), tensor(3, **I32)),
        lambda: B.adapters_torch(tensor(6, 64), tensor(6, 128), tensor(2, 8, 120), tensor(2, 64, 8), tensor(3, **I32)),
        lambda: B.adapters_torch(tensor(6, 64), tensor(6, 128), tensor(2, 8, 128), tensor(2, 60, 8), tensor(3, **I32)),
        lambda: B.adapters_torch(tensor(6, 64), tensor(6, 128), tensor(2, 8, 128), tensor(2, 64, 8), tensor(2, **I32)),
        lambda: B.adapters_torch(tensor(6, 64), tensor(6, 128), tensor(8, 128), tensor(64, 8), tensor(2, **I32)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert not calls, i


def test_the_refusal_of_a_gradient_names_the_call_that_takes_it(calls):
    for name, arg, back in (("route", "logits", "route_experts_backward_torch"), ("route", "bias", "route_experts_backward_torch"), ("gather", "x", "combine_rows_torch"),
                            ("combine", "x", "combine_rows_backward_torch"), ("combine", "weights", "combine_rows_backward_torch"), ("combine", "residual", "combine_rows_backward_torch")):
        with pytest.raises(ValueError, match=f"gradient is {back}"):
            one_of_each(change=lambda n, t, arg=arg: t.requires_grad_() if n == arg else t)[name]()
        assert callable(getattr(B, back))
    for name, arg in (("route back", "logits"), ("combine back", "dy"), ("adapters", "x")):
        with pytest.raises(ValueError, match="no gradient"):
            one_of_each(change=lambda n, t, arg=arg: t.requires_grad_() if n == arg else t)[name]()
    assert not calls
