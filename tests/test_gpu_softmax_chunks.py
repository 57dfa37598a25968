"""Softmax cross entropy where a logit is the sum of several chunks, each with an accumulator of its own (more than 512
columns), on the GPU. Bounds: operator_util."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import TYPES, check, inputs, softmax_reference  # noqa: E402

NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


# single CTAs and pairs, tiles of 128 and 256 classes; the last chunk whole, of one slice, of one column; odd and even numbers of
# chunks; more tiles than pairs of CTAs, so that a CTA's second tile begins with either accumulator
SIZES = [(1, 700, 1100), (40, 300, 1090), (129, 257, 577), (200, 100, 1600), (300, 700, 1025), (300, 700, 1536), (300, 700, 2049),
         (257, 1000, 3200), (2500, 3000, 1100), (2500, 3000, 2100), (100, 20000, 1200)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", SIZES)
def test_loss(ops, n, v, d, dtype):
    x, w, labels, _ = inputs(n, v, d, dtype, without=0.1 if n > 2 else 0.0)
    want = softmax_reference(x, w, labels)
    loss, lse = ops.softmax_loss(x, w, labels)
    check(loss, want["loss"], "loss")
    check(lse, want["lse"], "lse")


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", SIZES)
def test_gradients(ops, n, v, d, dtype):
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.1 if n > 2 else 0.0)
    want = softmax_reference(x, w, labels, weights, 0.5)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.5)):
        check(t, want[name], name)
