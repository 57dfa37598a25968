"""Gradients of so many classes that a piece has fewer rows than a tile of the products, on the GPU."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


# two pieces of 150 rows (pairs of CTAs), of 100 rows (single CTAs), and of 100 rows in single precision
@pytest.mark.parametrize("n,v,d,dtype", [(300, 20_000_000, 8, torch.bfloat16), (200, 40_000_000, 8, torch.bfloat16),
                                         (200, 40_000_000, 8, torch.float16), (200, 10_000_000, 5, torch.float32)], ids=str)
def test_pieces_give_what_their_rows_alone_give(ops, n, v, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    w = torch.randn(v, d, generator=g, device="cuda").to(dtype)
    labels = torch.randint(-1, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels[0], labels[n // 2 - 1], labels[n // 2], labels[n - 1] = v - 1, -1, 0, 1 << 23
    x[0, 0] = x[n // 2, 0] = 6.0  # (single precision: both halves have one scale)
    loss, lse, dx, dw = ops.softmax_loss_grad(x, w, labels, scale=2.0 ** 10)
    parts = [ops.softmax_loss_grad(x[a:a + n // 2], w, labels[a:a + n // 2], scale=2.0 ** 10) for a in (0, n // 2)]
    for k, t in enumerate((loss, lse, dx)):
        assert torch.equal(t, torch.cat([p[k] for p in parts]))
    # dW: one rounding each of the halves' and of the sum's (and of the fp32 sum)
    half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}[dtype]
    tiny = torch.finfo(dtype).smallest_normal * 2 * half
    for a in range(0, v, 4_000_000):
        q = [p[3][a:a + 4_000_000].double() for p in parts]
        off = (half + 2.0 ** -23) * (q[0].abs() + q[1].abs()) * 2.01 + 3 * tiny
        assert ((dw[a:a + 4_000_000].double() - q[0] - q[1]).abs() <= off).all()
    # and a few rows against 64 bits: logits of d products, exponentials and their sum, the logarithm
    for i in (0, n // 2, n - 1):
        logits = torch.cat([w[a:a + 4_000_000].double() @ x[i].double() for a in range(0, v, 4_000_000)])
        total = torch.logsumexp(logits, 0)
        off = (3 * d + 64) * 2.0 ** -23 * float(logits.abs().max() * d ** 0.5 + 20)
        assert abs(float(lse[i]) - float(total)) <= off and abs(float(loss[i]) - float(total - logits[int(labels[i])])) <= 2 * off
