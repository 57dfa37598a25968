"""Softmax cross entropy and its gradients where magnitudes are far from one, on the GPU. Bounds: operator_util."""
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


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n", [20, 300, 4096, 4097, 9000])
def test_weights_of_rows_without_a_label(ops, n, dtype):
    """They hold 2^60, infinities and NaN: no result depends on them, bit for bit. Some labels are beyond the last class."""
    x, w, labels, weights = inputs(n, 70, 40, dtype, without=0.3)
    labels[3], labels[n - 1], labels[n - 2], labels[5], labels[6] = 70, -1, -1, -1, 2
    without = (labels < 0) | (labels >= 70)
    held = weights.clone()
    held[without] = 2.0 ** 60
    held[5], held[n - 1] = float("inf"), float("nan")
    weights[without] = 1.0
    got = ops.softmax_loss_grad(x, w, labels, weights=held, scale=2.0 ** -10)
    want = softmax_reference(x, w, labels, weights, 2.0 ** -10)
    for name, t in zip(("loss", "lse", "dx", "dw"), got):
        check(t, want[name], name)
    assert all(torch.equal(s, t) for s, t in zip(got, ops.softmax_loss_grad(x, w, labels, weights=weights, scale=2.0 ** -10)))
