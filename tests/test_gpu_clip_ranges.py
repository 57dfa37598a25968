"""Clipping where norms and factors are near the ends of fp32's range, on the GPU."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("count", [2, 4, 9000])
def test_finite_elements_whose_norm_is_beyond_fp32(ops, count, in_place):
    """The norm is reported as infinity, and the elements stay as they are, those of the other tensors too."""
    t = [torch.full((count,), 3e38, device="cuda"), torch.randn(50, device="cuda").half(), torch.randn(700, device="cuda").bfloat16()]
    before = [x.clone() for x in t]
    out = None if in_place else [torch.zeros_like(x) for x in t]
    assert float(ops.clip_gradients(t, 1.0, out=out)) == math.inf
    assert all(torch.equal(a, b) for a, b in zip(t, before)) and all(torch.equal(a, b) for a, b in zip(out or t, before))


def test_the_largest_norm_that_fp32_holds(ops):
    """Half of fp32's range each way: still clipped."""
    t = torch.full((4,), 2.0 ** 126, device="cuda")
    assert float(ops.clip_gradients([t], 2.0 ** 100)) == 2.0 ** 127
    assert torch.equal(t, torch.full((4,), 2.0 ** 99, device="cuda"))


@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-6])
@pytest.mark.parametrize("size", [1e30, 1e34, 3e36])
def test_factors_below_the_normal_range_of_fp32(ops, size, max_norm):
    """The norm's error (2^-21), the factor's and the product's roundings (2^-24 each), and results of the type's smallest steps."""
    g = torch.Generator(device="cuda").manual_seed(5)
    t = [torch.randn(1000, generator=g, device="cuda") * size, (torch.randn(900, generator=g, device="cuda") * size).bfloat16()]
    before = [x.double() for x in t]
    norm = math.sqrt(sum(float((b * b).sum()) for b in before))
    assert norm < 3e38
    got = ops.clip_gradients(t, max_norm)
    assert abs(float(got) - norm) <= 2.0 ** -21 * norm
    for b, x, half in zip(before, t, (2.0 ** -24, 2.0 ** -8)):
        want = b * (max_norm / (norm + 1e-6))
        assert ((x.double() - want).abs() <= want.abs() * (2.0 ** -21 + 3 * 2.0 ** -24 + half * (1 + 2.0 ** -20)) + 2.0 ** -126 * 2 * half).all()
