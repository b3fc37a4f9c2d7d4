"""The bounds on products of codes as a whole, without a GPU: what they accept and what they see."""
import numpy as np
import pytest

from oracle import operators as O


def operands(kind, M=64, N=330, K=1100, seed=0):
    """Codes and scales of a product: normal values; one value of each block a hundred times the others; all positive, with one thirty times."""
    rng = np.random.default_rng(seed)
    a = rng.normal(size=(M, K)) * np.exp(0.5 * rng.normal(size=(M, 1)))
    b = rng.normal(size=(N, K)) * 0.05
    if kind == "outliers":
        a[:, 5::128] *= 100
    if kind == "positive":
        a, b = np.abs(a), np.abs(b)
        a[:, 77::128] *= 30
    return O.quantize(a.astype(np.float32), 1) + O.quantize(b.astype(np.float32), 128)


KINDS = ["normal", "outliers", "positive"]


@pytest.mark.parametrize("ytype", ["f16", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("K", [128, 300, 1100, 4096])
def test_the_aggregate_bound_takes_what_is_right_and_sees_what_is_wrong(kind, ytype, K):
    ca, sa, cb, sb = operands(kind, K=K)
    N = cb.shape[0]
    ref = O.values(ca, sa, 1) @ O.values(cb, sb, 128).T
    model = O.core_sums(ca, sa, cb, sb)
    off = lambda z: O.aggregate(O.nearest(z, ytype), ref, model, ytype)  # noqa: E731
    assert off(ref) <= 1 and off(model) <= 1
    for wrong in (ref * 1.005, ref * 0.995, ref * 1.001):
        assert off(wrong) > 1
    # (a thousandth of the result left out at random; the last column; one of 16 weight columns' scales)
    assert off(ref + 1e-3 * np.sqrt((ref ** 2).mean()) * np.random.default_rng(1).normal(size=ref.shape)) > 1
    assert off(O.values(ca, sa, 1)[:, :-1] @ O.values(cb, sb, 128)[:, :-1].T) > 1
    swapped = sb.copy()
    swapped[0], swapped[1] = sb[1], sb[0]
    assert off(O.values(ca, sa, 1) @ O.values(cb, swapped, 128).T) > 1
    if K > 128:
        # blocks added up in bf16
        part = np.zeros_like(ref)
        for k in range(0, K, 128):
            s = slice(k, k + 128)
            part = O.nearest(part + O.values(ca, sa, 1)[:, s] @ O.values(cb, sb, 128)[:, s].T, "bf16")
        assert O.aggregate(O.nearest(part, ytype), ref, model, ytype) > 1
        assert off(O.values(ca, np.roll(sa, 1, 1), 1) @ O.values(cb, sb, 128).T) > 1


@pytest.mark.parametrize("kind,least,most", [("normal", 1e-5, 4e-5), ("outliers", 1e-5, 1.2e-4), ("positive", 1e-6, 3e-5)])
def test_the_model_of_the_cores_stays_below_the_rounding_of_16_bits(kind, least, most):
    """A rounding to f16 is 2e-4 of the result, to bf16 1.6e-3."""
    ca, sa, cb, sb = operands(kind)
    ref = O.values(ca, sa, 1) @ O.values(cb, sb, 128).T
    off = np.sqrt(((O.core_sums(ca, sa, cb, sb) - ref) ** 2).mean() / (ref ** 2).mean())
    assert least < off < most
