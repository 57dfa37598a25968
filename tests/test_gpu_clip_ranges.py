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
