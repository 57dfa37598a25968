"""Softmax cross entropy and its gradients against 64 bits, on the GPU. Bounds: operator_util."""
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


# one row and one class; tiles' edges (128 rows, 256 and 128 classes, 64 columns) and around them; odd sizes; many row tiles;
# few rows and many classes (the sum over classes is cut); many rows and few classes (the sum over rows is cut)
SIZES = [(1, 1, 1), (1, 2, 16), (3, 5, 7), (128, 256, 64), (129, 257, 65), (127, 255, 63), (64, 128, 128), (300, 700, 100),
         (1, 5000, 96), (17, 9001, 72), (2000, 10, 33), (1500, 1300, 264)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", SIZES)
def test_loss(ops, n, v, d, dtype):
    x, w, labels, _ = inputs(n, v, d, dtype)
    want = softmax_reference(x, w, labels)
    loss, lse = ops.softmax_loss(x, w, labels)
    check(loss, want["loss"], "loss")
    check(lse, want["lse"], "lse")


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", SIZES)
def test_gradients(ops, n, v, d, dtype):
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.2 if n > 2 else 0.0)
    scale = 0.5
    want = softmax_reference(x, w, labels, weights, scale)
    loss, lse, dx, dw = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=scale)
    for name, got in (("loss", loss), ("lse", lse), ("dx", dx), ("dw", dw)):
        check(got, want[name], name)
    assert dx.dtype == dtype and dw.dtype == dtype


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n", [4096, 4097, 9000])
def test_weights_of_very_different_size(ops, n, dtype):
    """One weight 2^12 times the others, at the end: P's scale goes by the largest, few weights and many."""
    x, w, labels, weights = inputs(n, 70, 40, dtype, without=0.1)
    weights[-1] = 2.0 ** 12
    labels[-1] = 3
    want = softmax_reference(x, w, labels, weights, 2.0 ** -20)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights, scale=2.0 ** -20)):
        check(t, want[name], name)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_equal_inputs_give_equal_bits(ops, dtype):
    x, w, labels, weights = inputs(700, 3000, 200, dtype, without=0.1)
    a = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.01)
    b = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.01)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_strides_and_alignment(ops, dtype):
    """Rows of a wider matrix, at an odd offset: the same results as from contiguous copies."""
    x, w, labels, weights = inputs(150, 333, 72, dtype)
    wide_x = torch.full((150, 99), float("nan"), dtype=dtype, device="cuda")
    wide_w = torch.full((333, 81), float("nan"), dtype=dtype, device="cuda")
    wide_x[:, 5:77] = x
    wide_w[:, 3:75] = w
    for f in (lambda a, b: ops.softmax_loss(a, b, labels), lambda a, b: ops.softmax_loss_grad(a, b, labels, weights=weights)):
        for s, t in zip(f(x, w), f(wide_x[:, 5:77], wide_w[:, 3:75])):
            assert torch.equal(s, t)
    aligned = torch.zeros(150, 160, dtype=dtype, device="cuda")
    aligned[:, 64:136] = x
    for s, t in zip(ops.softmax_loss(x, w, labels), ops.softmax_loss(aligned[:, 64:136], w, labels)):
        assert torch.equal(s, t)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_rows_without_a_label(ops, dtype):
    """They hold infinities and NaN: nothing of them may reach any result. One batch has no label at all."""
    x, w, labels, weights = inputs(260, 500, 80, dtype, without=0.3)
    x[labels < 0] = float("nan")
    x[(labels < 0).nonzero()[0]] = float("inf")
    clean = torch.where((labels >= 0)[:, None], x, torch.zeros_like(x))
    got = ops.softmax_loss_grad(x, w, labels, weights=weights)
    want = softmax_reference(clean, w, labels, weights)
    for name, t in zip(("loss", "lse", "dx", "dw"), got):
        check(t, want[name], name)
    none = torch.full_like(labels, -1)
    for t in ops.softmax_loss(x, w, none) + ops.softmax_loss_grad(x, w, none, weights=weights):
        assert not t.any()


def test_labels_beyond_the_last_class(ops):
    x, w, labels, _ = inputs(40, 30, 24, torch.bfloat16)
    bad = labels.clone()
    bad[7] = 30
    bad[9] = 2 ** 31 - 1
    without = labels.clone()
    without[[7, 9]] = -1
    for f in (ops.softmax_loss, ops.softmax_loss_grad):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got, want = f(x, w, bad, status=status), f(x, w, without)
        assert int(status) == ops.STATUS_BAD_ID
        assert all(torch.equal(s, t) for s, t in zip(got, want))
        status.zero_()
        f(x, w, labels, status=status)
        assert int(status) == 0


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_confident_rows(ops, dtype):
    """Logits of +-60: losses near zero and near 100, probabilities far below the types' smallest steps."""
    g = torch.Generator(device="cuda").manual_seed(3)
    n, v, d = 200, 400, 64
    w = torch.randn(v, d, generator=g, device="cuda")
    w = (w / w.norm(dim=1, keepdim=True)).to(dtype)
    labels = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    x = (w[labels.long()].float() * 60 * torch.where(torch.arange(n, device="cuda") % 3 == 0, -1.0, 1.0)[:, None]).to(dtype)
    want = softmax_reference(x, w, labels)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels)):
        check(t, want[name], name)


def test_gradients_against_differences(ops):
    """Directional derivatives in fp32: central differences, h = 2^-6. The third derivative of the loss along a direction u with
    logits' change z is at most 2 max|z|^3 per row, so the difference is off by h^2 / 3 max|z|^3 per unit weight, and by the
    losses' rounding over h."""
    x, w, labels, weights = inputs(50, 40, 24, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(9)
    u, t = torch.randn(x.shape, generator=g, device="cuda"), torch.randn(w.shape, generator=g, device="cuda") * 0.2
    loss, _, dx, dw = ops.softmax_loss_grad(x, w, labels, weights=weights)
    h = 2.0 ** -6
    total = float(weights.double().sum())
    rounding = float((weights.double() * 2 * softmax_reference(x, w, labels)["loss"][1]).sum()) / h
    for du, dt, slope in ((u, 0 * t, (dx.double() * u).sum()), (0 * u, t, (dw.double() * t).sum())):
        plus, minus = (ops.softmax_loss(x + s * du, w + s * dt, labels)[0].double() for s in (h, -h))
        diff = ((plus - minus) * weights.double()).sum() / (2 * h)
        z = (du.double() @ w.double().T + x.double() @ dt.double().T).abs().max()
        assert abs(float(diff - slope)) <= total * h * h / 3 * float(z) ** 3 + rounding + 1e-4 * abs(float(slope))


def test_no_rows(ops):
    w = torch.randn(9, 16, device="cuda", dtype=torch.bfloat16)
    x, y = w[:0], torch.empty(0, dtype=torch.int32, device="cuda")
    loss, lse = ops.softmax_loss(x, w, y)
    assert loss.numel() == 0 and lse.numel() == 0
    loss, lse, dx, dw = ops.softmax_loss_grad(x, w, y)
    assert dx.shape == (0, 16) and dw.shape == (9, 16) and not dw.any()


def test_on_another_stream_and_captured(ops):
    x, w, labels, weights = inputs(400, 900, 128, torch.bfloat16, without=0.1)
    want = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.1, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    # two graphs of the same call, replayed one behind the other and on two streams at once
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.1))
        graphs.append(graph)
    x2 = x.clone()
    x.copy_(x2.flip(0))
    want2 = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.1)
    torch.cuda.synchronize()
    for graph, stream in zip(graphs, (torch.cuda.Stream(), torch.cuda.Stream())):
        with torch.cuda.stream(stream):
            graph.replay()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(s, t) for s, t in zip(out, want2))


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_many_passes_on_two_streams(ops, dtype):
    """Captured passes one behind the other on two streams at once: the kernels of one follow those of the other on the same SMs.
    No wait runs out, and every pass gives the bits of the first."""
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    batches = [inputs(700, 1300, 200, dtype, seed=k, without=0.1) for k in range(2)]
    first = [ops.softmax_loss_grad(*b[:3], weights=b[3], status=status) for b in batches]
    torch.cuda.synchronize()
    graphs, last = [], []
    for b in batches:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(10):
                out = ops.softmax_loss_grad(*b[:3], weights=b[3], status=status)
        graphs.append(graph)
        last.append(out)
    streams = [torch.cuda.Stream() for _ in batches]
    for _ in range(20):
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    assert int(status) == 0
    assert all(torch.equal(s, t) for a, b in zip(first, last) for s, t in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=NAMES.get)
def test_several_pieces(ops, dtype):
    """So many classes that the rows are taken in pieces: dW is summed over them."""
    n, v, d = 5000, 150001 if dtype == torch.bfloat16 else 60001, 24
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.05)
    want = softmax_reference(x, w, labels, weights, 1.0 / n)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights, scale=1.0 / n)):
        check(t, want[name], name)


def test_weights_beyond_32_bit_offsets(ops):
    """2.2 G elements of W, labels at both ends: loss, dX, and rows of dW around element 2^31."""
    n, v, d = 3, 530000, 4096
    g = torch.Generator(device="cuda").manual_seed(4)
    w = torch.empty(v, d, dtype=torch.bfloat16, device="cuda")
    for a in range(0, v, 53000):
        w[a:a + 53000] = (torch.randn(53000, d, generator=g, device="cuda") / 32).bfloat16()
    x = torch.randn(n, d, generator=g, device="cuda").bfloat16()
    labels = torch.tensor([0, 2 ** 19, v - 1], dtype=torch.int32, device="cuda")
    loss, lse, dx, dw = ops.softmax_loss_grad(x, w, labels)
    assert all(torch.equal(s, t) for s, t in zip(ops.softmax_loss(x, w, labels), (loss, lse)))
    X = x.double()
    logits = torch.cat([X @ w[a:a + 53000].double().T for a in range(0, v, 53000)], 1)
    total = torch.logsumexp(logits, 1)
    mine = logits.gather(1, labels.long()[:, None])[:, 0]
    # logits of 4096 products of magnitude 1/32 on average: the worst case of their sums (operator_util), and the largest logit's rounding
    off = d * 2.0 ** -23 * float((X.abs() @ w[:53000].double().abs().T).max()) * 1.2 + 2.0 ** -18
    assert ((lse.double() - total).abs() <= off).all() and ((loss.double() - (total - mine)).abs() <= 2 * off).all()
    p = (logits - total[:, None]).exp()
    p[torch.arange(n), labels.long()] -= 1.0
    want = sum(p[:, a:a + 53000] @ w[a:a + 53000].double() for a in range(0, v, 53000))
    # the label's row of W decides: P's rounding and the result's, and the logits' error
    assert ((dx.double() - want).abs() <= (2.0 ** -8 + 4 * off) * (p.abs().max(1, keepdim=True).values * 0.2 + want.abs())).all()
    for c in (0, 1, 2 ** 19 - 1, 2 ** 19, 2 ** 19 + 1, v - 2, v - 1):
        ref = p[:, c] @ X
        assert ((dw[c].double() - ref).abs() <= (2.0 ** -7 + 4 * off) * (p[:, c].abs() @ X.abs())).all()


def test_loss_of_many_rows(ops):
    """So many rows that the loss takes them in pieces: rows around the pieces' ends."""
    n, v, d = 180000, 100000, 16
    x, w, labels, _ = inputs(n, v, d, torch.bfloat16, without=0.1)
    loss, lse = ops.softmax_loss(x, w, labels)
    piece = (1 << 30) // (8 * 2 * -(-v // 256)) // 256 * 256  # pairs of floats, two per tile of 256 classes
    assert 4096 < piece < n
    rows = torch.cat([torch.arange(0, 60), torch.arange(piece - 60, piece + 60), torch.arange(n - 60, n)]).cuda()
    want = softmax_reference(x[rows], w, labels[rows])
    check(loss[rows], want["loss"], "loss")
    check(lse[rows], want["lse"], "lse")


def test_refusals(ops):
    x, w, labels, weights = inputs(8, 6, 16, torch.float32)
    bad = [
        lambda: ops.softmax_loss(x.bfloat16(), w, labels),
        lambda: ops.softmax_loss(x[:, :8], w, labels),
        lambda: ops.softmax_loss(x, w[:0], labels),
        lambda: ops.softmax_loss(x.cpu(), w, labels),
        lambda: ops.softmax_loss(x.double(), w.double(), labels),
        lambda: ops.softmax_loss(x, w, labels.long()),
        lambda: ops.softmax_loss(x, w, labels[:-1]),
        lambda: ops.softmax_loss(x.T.contiguous().T, w, labels),
        lambda: ops.softmax_loss(x[:1].expand(8, 16), w, labels),
        lambda: ops.softmax_loss_grad(x, w, labels, weights=weights[:3]),
        lambda: ops.softmax_loss_grad(x, w, labels, scale=float("nan")),
        lambda: ops.softmax_loss_grad(x, w, labels, weights=weights.double()),
        lambda: ops.softmax_loss(x, w, labels, status=torch.zeros(2, dtype=torch.int32, device="cuda")),
    ]
    for f in bad:
        with pytest.raises((ValueError, ops.ChicleError)):
            f()
