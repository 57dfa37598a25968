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


@pytest.mark.parametrize("size_x,size_w", [(1e-18, 1e-18), (1e-25, 1e-25), (1e-30, 1e30), (1e30, 1e-30), (1e-35, 1e-35)])
@pytest.mark.parametrize("n,v", [(40, 257), (300, 257), (300, 100), (20, 3), (300, 512)])
def test_single_precision_of_far_sizes(ops, n, v, size_x, size_w):
    """Operands far below (and above) one, blocks of classes that are not full: the scales' product leaves fp32's range, the
    results do not."""
    x, w, labels, weights = inputs(n, v, 72, torch.float32, without=0.1)
    x, w = x * size_x, w * size_w
    want = softmax_reference(x, w, labels, weights, 1.0)
    loss, lse = ops.softmax_loss(x, w, labels)
    check(loss, want["loss"], "loss")
    check(lse, want["lse"], "lse")
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights)):
        check(t, want[name], name)


@pytest.mark.parametrize("n,v", [(40, 257), (300, 300)])
def test_single_precision_of_large_operands_with_logits_of_zero(ops, n, v):
    """x and w of 1e25 without a column in common: all logits are 0, the loss log(v) (rounded: 2^-20), and the gradients a mean of
    rows, off by their planes and the sums of 3 v and 3 n products."""
    x, w, labels, _ = inputs(n, v, 80, torch.float32)
    x, w = x * 1e25, w * 1e25
    x[:, 40:], w[:, :40] = 0.0, 0.0
    loss, lse, dx, dw = ops.softmax_loss_grad(x, w, labels, scale=1.0 / n)
    for t in (loss, lse) + ops.softmax_loss(x, w, labels):
        assert ((t.double() - torch.tensor(float(v), dtype=torch.float64).log().item()).abs() <= 2.0 ** -20).all()
    p = torch.full((n, v), 1.0 / v, dtype=torch.float64, device="cuda")
    p[torch.arange(n), labels.long()] -= 1.0
    p /= n
    for got, a, b, k in ((dx, p, w.double(), v), (dw, p.T, x.double(), n)):
        off = (3 * k + 32) * 2.0 ** -23 * (a.abs() @ b.abs()) + 2.0 ** -38 * a.abs().sum(1, keepdim=True) * b.abs().max()
        assert ((got.double() - a @ b).abs() <= off).all()


@pytest.mark.parametrize("dtype", TYPES[1:], ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", [(40, 300, 64), (300, 700, 1100)])
def test_classes_with_a_logit_of_minus_infinity(ops, n, v, d, dtype):
    """Rows of x above zero, two classes of -inf (one of them all that its block holds but for another): their probability is 0; a row
    with such a label has an infinite loss."""
    x, w, labels, weights = inputs(n, v, d, dtype)
    x = x.abs() + 0.125
    w[:, 1:] *= 0.25
    gone = [5, v - 1]
    stay = [k for k in range(v) if k not in gone]
    labels = torch.where((labels == 5) | (labels == v - 1), torch.full_like(labels, 6), labels)
    w[gone] = -float("inf")
    at = torch.tensor([stay.index(int(k)) for k in labels.tolist()], dtype=torch.int32, device="cuda")
    want = softmax_reference(x, w[stay], at, weights)
    for out in (ops.softmax_loss(x, w, labels), ops.softmax_loss_grad(x, w, labels, weights=weights)):
        check(out[0], want["loss"], "loss")
        check(out[1], want["lse"], "lse")
    check(out[3][stay], want["dw"], "dw")
    assert not out[3][gone].any()
    labels[3] = 5
    for out in (ops.softmax_loss(x, w, labels), ops.softmax_loss_grad(x, w, labels)):
        assert out[0][3] == float("inf") and torch.isfinite(out[0][:3]).all() and torch.isfinite(out[1]).all()
