"""How exact the softmax gradients are over long sums, norm by norm, on the GPU.

The element-wise bounds of operator_util are worst cases that grow with the length of a sum. Here the error's norm is held to what
the kernels' design gives, so that a lost chunk, plane or rounding shows.

Single precision: an accumulator takes 512 terms of each of three products of planes, in 96 steps of 16 terms, and a step cuts off at
most a unit in the last place of the accumulator, 2^-23 of it, in the mean half of one, 2^-24.5 of it (units are 2^-24 to 2^-23 of a number).
Sums of one sign: 96 2^-23 of a chunk's sum at worst; the chunks are added in fp32 (k / 512 roundings of 2^-24 of the sum); planes,
the product of planes that is left out, exponentials and logits: 6 times 2^-20 in all. An accumulator for all k terms would cut off
3 k / 16 times 2^-24.5 of a sum that grows from 0: half of that, 1.4e-4 at 60 000 terms.
Sums of both signs: the mean of the steps, 96 2^-24.5, and 2^-20 for the rest, of the result's norm. One product of planes less would
leave 2^-12 of every term.

16 bits: the result's rounding and that of P's entries, half a step at most and uniform below it: half / sqrt(3) in the mean, sqrt(2)
times that for the two together (entries of the label are most of P; the weights spread them over all mantissas); a tenth for
everything else. The loss as in single precision.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import HALF, TYPES  # noqa: E402

MEAN = 96 * 2.0 ** -24.5 + 2.0 ** -20
NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


def exact(x, w, labels, scale, weights=None):
    X, W = x.double(), w.double()
    logits = X @ W.T
    p = torch.softmax(logits, 1)
    loss = torch.logsumexp(logits, 1) - logits.gather(1, labels.long()[:, None])[:, 0]
    p[torch.arange(len(p), device=p.device), labels.long()] -= 1.0
    p *= scale if weights is None else weights.double()[:, None] * scale
    return loss, p, p @ W, p.T @ X


def case(n, v, d, dtype, shift):
    """Logits of order one whatever the shift: x is small where w has a mean."""
    g = torch.Generator(device="cuda").manual_seed(21)
    x = (torch.randn(n, d, generator=g, device="cuda") / d ** 0.5 + (shift if v < n else 0.0)).to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda") / (d ** 0.5 if v < n else 1.0) + (shift if v > n else 0.0)).to(dtype)
    labels = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    return x, w, labels


def off(got, want, scale_norm):
    return float((got.double() - want).norm() / scale_norm)


# dX sums over many classes, dW over many rows; the second two with about as many tiles as pairs of CTAs, so that sums are not cut
# for the SMs' sake and chunks alone keep accumulators short
LONG = [(4352, 60000, 1024), (50000, 4608, 1024)]


@pytest.mark.parametrize("n,v,d", [(96, 60000, 64), (48000, 40, 64)] + LONG)
def test_sums_of_one_sign_in_single_precision(ops, n, v, d):
    x, w, labels = case(n, v, d, torch.float32, 3.0)
    _, p, dx, dw = exact(x, w, labels, 1.0)
    _, _, gx, gw = ops.softmax_loss_grad(x, w, labels)
    k = max(n, v)
    bound = 96 * 2.0 ** -23 + k / 512 * 2.0 ** -24 + 6 * 2.0 ** -20
    for got, want, a, b in ((gx, dx, p, w.double()), (gw, dw, p.T, x.double())):
        assert off(got, want, (a.abs() @ b.abs()).norm()) <= bound


@pytest.mark.parametrize("n,v,d", [(300, 20000, 96), (20000, 300, 96), (2000, 3000, 700)] + LONG)
def test_sums_of_both_signs_in_single_precision(ops, n, v, d):
    x, w, labels = case(n, v, d, torch.float32, 0.0)
    loss, _, dx, dw = exact(x, w, labels, 1.0 / n)
    got, _, gx, gw = ops.softmax_loss_grad(x, w, labels, scale=1.0 / n)
    for s, t in ((got, loss), (gx, dx), (gw, dw)):
        assert off(s, t, t.norm()) <= MEAN


@pytest.mark.parametrize("dtype", TYPES[1:], ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", [(20, 3000, 96), (300, 20000, 96), (20000, 300, 96), (2000, 3000, 1100)])
def test_both_signs_in_16_bits(ops, n, v, d, dtype):
    """Up to 32 rows P has two planes, and the result's rounding is what is left."""
    x, w, labels = case(n, v, d, dtype, 0.0)
    weights = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda") + 0.5
    loss, _, dx, dw = exact(x, w, labels, 1.0, weights)
    got, _, gx, gw = ops.softmax_loss_grad(x, w, labels, weights=weights)  # (scale 1: far from fp16's subnormals)
    assert off(got, loss, loss.norm()) <= MEAN
    roundings = 1.0 if n <= 32 else 2.0 ** 0.5
    for s, t in ((gx, dx), (gw, dw)):
        assert off(s, t, t.norm()) <= 1.1 * roundings * HALF[dtype] / 3 ** 0.5


@pytest.mark.parametrize("dtype", TYPES[1:], ids=NAMES.get)
def test_very_many_classes_of_one_sign(ops, dtype):
    """What accumulators cut off has one sign, so it shows in the mean error: an eighth of half a step of the sums' magnitudes at
    most. Beside it the roundings' mean: of P's entry of the label, one per row (half / sqrt(3) of half of the magnitudes, the mean of
    32 rows, three times that), of the results (of 32 x 1024 of them: nothing)."""
    n, v, d, step = 2048, 3_000_000, 1024, 100_000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.randn(n, d, generator=g, device="cuda") / d ** 0.5).to(dtype)
    w = torch.empty(v, d, dtype=dtype, device="cuda")
    for a in range(0, v, step):
        w[a:a + step] = (torch.randn(step, d, generator=g, device="cuda") + 3.0).to(dtype)
    labels = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.rand(n, generator=g, device="cuda") + 0.5
    dx = ops.softmax_loss_grad(x, w, labels, weights=weights)[2]
    rows = torch.arange(0, n, n // 32, device="cuda")
    X = x[rows].double()
    p = torch.softmax(torch.cat([X @ w[a:a + step].double().T for a in range(0, v, step)], 1), 1)
    p[torch.arange(len(rows)), labels[rows].long()] -= 1.0
    p *= weights[rows].double()[:, None]
    want, size = torch.zeros_like(X), torch.zeros_like(X)
    for a in range(0, v, step):
        b = w[a:a + step].double()
        want += p[:, a:a + step] @ b
        size += p[:, a:a + step].abs() @ b.abs()
    mean = float(((dx[rows].double() - want) / size).mean())
    assert abs(mean) <= HALF[dtype] * (1 / 8 + 3 * 0.5 / 3 ** 0.5 / 32 ** 0.5), mean


@pytest.mark.parametrize("dtype", TYPES[1:], ids=NAMES.get)
def test_very_many_rows_of_one_sign(ops, dtype):
    """The same of dW: an eighth, and the results' roundings (of 16 x 64 of them, three times their mean)."""
    n, v, d = 4_000_000, 16, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    x = (torch.randn(n, d, generator=g, device="cuda") / 8 + 3.0).to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda") / 8).to(dtype)
    labels = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.rand(n, generator=g, device="cuda") + 0.5
    scale = 2.0 ** -14
    dw = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=scale)[3]
    want, size = torch.zeros(v, d, dtype=torch.float64, device="cuda"), torch.zeros(v, d, dtype=torch.float64, device="cuda")
    for a in range(0, n, 500_000):
        _, p, _, part = exact(x[a:a + 500_000], w, labels[a:a + 500_000], scale, weights[a:a + 500_000])
        want += part
        size += p.abs().T @ x[a:a + 500_000].double().abs()
    mean = float(((dw.double() - want) / size).mean())
    assert abs(mean) <= HALF[dtype] * (1 / 8 + 3 / 3 ** 0.5 / 1024 ** 0.5), mean


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", [(1, 3000, 4096), (300, 700, 4096), (300, 700, 1000)])
def test_logits_of_one_sign(ops, n, v, d, dtype):
    """An accumulator of a logit takes 64 steps (single precision: 32 that count, the small products of planes come first); a step cuts
    off 1.6e-7 of it, of a growing sum half of that: 64 x 1.6e-7 / 2 = 5.1e-6 of the logit; chunks, planes, exponentials: 2^-20."""
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(n, d, generator=g, device="cuda").abs().to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda").abs() / 8).to(dtype)
    labels = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    logits = x.double() @ w.double().T
    want = torch.logsumexp(logits, 1)
    own = logits.gather(1, labels.long()[:, None])[:, 0]
    bound = 5.1e-6 + 2.0 ** -20
    for out in (ops.softmax_loss(x, w, labels), ops.softmax_loss_grad(x, w, labels)):
        assert ((out[1].double() - want).abs() <= bound * want).all()
        assert ((out[0].double() - (want - own)).abs() <= bound * want).all()
