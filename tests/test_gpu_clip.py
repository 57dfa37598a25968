"""The norm over many tensors and clipping against 64 bits, on the GPU, and a step of a softmax model with all operators."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import HALF, TYPES, softmax_reference  # noqa: E402

NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}
# squares are added eight at a time in fp32: 8 roundings of the sum, half of that on the norm, and the norm's own
NORM = 2.0 ** -21


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


def check(ops, tensors, max_norm, out=None):
    before = [t.clone() for t in tensors]
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in before))
    got = ops.clip_gradients(tensors, max_norm, out=out)
    assert abs(float(got) - norm) <= NORM * norm
    f = min(1.0, max_norm / (norm + 1e-6))
    for b, t, o in zip(before, tensors, out or tensors):
        want = b.double() * f
        # the factor's error (the norm's, rounded to fp32), the product's rounding, the type's
        off = want.abs() * (NORM + 3 * 2.0 ** -24 + HALF[b.dtype] * (1 + NORM)) + torch.finfo(b.dtype).smallest_normal * 2 * HALF[b.dtype]
        assert ((o.double() - want).abs() <= off).all()
        if f == 1.0:
            assert torch.equal(o, b)
        if out is not None:
            assert torch.equal(t, b)


@pytest.mark.parametrize("factor", [0.3, 1.5])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_sizes(ops, dtype, in_place, factor):
    sizes = [1, 7, 0, 8, 8191, 8192, 8193, 100003, 64]
    tensors = [torch.randn(k, device="cuda").to(dtype) for k in sizes]
    out = None if in_place else [torch.full_like(t, 9.0) for t in tensors]
    check(ops, tensors, factor * math.sqrt(sum(sizes)), out)


@pytest.mark.parametrize("shift", [0, 1])
def test_pieces_of_flat_buffers(ops, shift):
    """Every alignment, in and out at the same and at different places within 16 bytes; the elements around are left alone."""
    sizes = [3, 10000, 5, 17, 9001, 1]
    flat = torch.randn(sum(sizes) + 3, device="cuda").bfloat16()
    to = torch.full((sum(sizes) + 8,), 5.0, device="cuda").bfloat16()
    check(ops, list(torch.split(flat[1:-2], sizes)), 3.0, list(torch.split(to[1 + shift:1 + shift + sum(sizes)], sizes)))
    assert (to[:1 + shift] == 5).all() and (to[1 + shift + sum(sizes):] == 5).all()


def test_mixed_types_and_many_tensors(ops):
    """More than one launch takes (512), types mixed, shapes of several dimensions."""
    g = torch.Generator(device="cuda").manual_seed(1)
    tensors = [torch.randn(3, 5 + k % 7, generator=g, device="cuda").to(TYPES[k % 3]) for k in range(1300)]
    check(ops, tensors, 2.0)
    check(ops, tensors[:3], 100.0)
    check(ops, [torch.randn(5, device="cuda")] + [torch.randn(70000, device="cuda") for _ in range(600)], 1.0)


@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e15, 1e25])
def test_far_magnitudes(ops, size):
    """Squares beyond fp32's range on either side."""
    check(ops, [torch.randn(10007, device="cuda") * size, torch.zeros(5, device="cuda")], 1.0)


def test_zeros_and_zero_norm(ops):
    check(ops, [torch.zeros(100, device="cuda")], 1.0)
    t = [torch.randn(100, device="cuda")]
    check(ops, t, 0.0)
    assert not t[0].any()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_norms_that_are_not_finite(ops, value):
    t = [torch.randn(9000, device="cuda"), torch.randn(50, device="cuda").half()]
    t[0][5000] = value
    before = [x.clone() for x in t]
    norm = float(ops.clip_gradients(t, 1.0))
    assert not math.isfinite(norm)
    assert all(torch.equal(a.nan_to_num(7), b.nan_to_num(7)) for a, b in zip(t, before))


def test_norm_alone_and_captured(ops):
    t = [torch.randn(30000, device="cuda"), torch.randn(11, device="cuda")]
    keep = [x.clone() for x in t]
    a = float(ops.clip_gradients(t, math.inf))
    assert all(torch.equal(x, y) for x, y in zip(t, keep))
    out = [torch.empty_like(x) for x in t]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = ops.clip_gradients(t, 1.0, out=out)
    for x in t:
        x.mul_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    assert abs(float(norm) - 3 * a) <= 4 * NORM * 3 * a
    eager = [torch.empty_like(x) for x in t]
    ops.clip_gradients(t, 1.0, out=eager)
    assert all(torch.equal(x, y) for x, y in zip(out, eager))


def test_neighbours_and_streams(ops):
    """Pieces of one buffer next to each other, given as an iterator, on another stream; the same tensor twice for its norm alone."""
    flat = torch.randn(20000, device="cuda")
    want = [flat.clone() for _ in range(2)]
    n = float(ops.clip_gradients([want[0][:7], want[0][7:]], 1.0))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m = ops.clip_gradients((flat[a:b] for a, b in ((0, 7), (7, 20000))), 1.0, stream=side.cuda_stream)
    side.synchronize()
    assert float(m) == n and torch.equal(flat, want[0])
    # (in place, and the pieces in the other order: the same sum in another order of its parts)
    ops.clip_gradients([want[1][7:], want[1][:7]], 1.0)
    assert torch.allclose(want[1], want[0], rtol=4 * NORM, atol=0)


def test_refusals(ops):
    t = torch.randn(8, 8, device="cuda")
    for f in (lambda: ops.clip_gradients([], 1.0), lambda: ops.clip_gradients([t], -1.0), lambda: ops.clip_gradients([t], float("nan")),
              lambda: ops.clip_gradients([t.T[1:]], 1.0), lambda: ops.clip_gradients([t.cpu()], 1.0), lambda: ops.clip_gradients([t.double()], 1.0),
              lambda: ops.clip_gradients([t], 1.0, out=[t.half()]), lambda: ops.clip_gradients([t], 1.0, out=[]),
              lambda: ops.clip_gradients([t[:4]], 1.0, out=[t[1:5]]), lambda: ops.clip_gradients([t, t], 1.0),
              lambda: ops.clip_gradients([t[:5], t[4:]], 1.0), lambda: ops.clip_gradients([t[:2], t[2:4]], 1.0, out=[t[4:6], t[4:6]]),
              lambda: ops.clip_gradients([t[:2], t[2:4]], 1.0, out=[t[4:6], t[1:3]])):
        with pytest.raises((ValueError, ops.ChicleError)):
            f()


def test_a_training_step(ops):
    """Look vectors up, take the loss and its gradients, sum the vectors' gradient by id into the shared table's, clip all; in
    single precision against 64 bits. The bound: each operator's own on its computed inputs, so the last is compared with
    the definition applied to what the ones in front gave, and the whole chain within 1e-5 of the largest gradient (losses'
    bounds at these sizes: logits of 6 x 40 products, 3e-5 x 1/3 of their magnitudes at worst, a hundredth of that on average)."""
    g = torch.Generator(device="cuda").manual_seed(2)
    v, d, n = 300, 40, 500
    table = torch.randn(v, d, generator=g, device="cuda") * 0.3
    ids = torch.randint(-1, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.randint(-1, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    bias = torch.randn(d, generator=g, device="cuda") * 0.1
    x = ops.embedding(table, ids, scale=2.0) + bias
    loss, lse, dx, dtable = ops.softmax_loss_grad(x, table, labels, scale=1.0 / n)
    ops.embedding_grad(ids, dx, v, scale=2.0, out=dtable, accumulate=True)
    dbias = dx.sum(0)
    norm = ops.clip_gradients([dtable, dbias], 0.01)

    T = table.double().requires_grad_()
    B = bias.double().requires_grad_()
    rows = torch.where((ids >= 0)[:, None], T[ids.clamp(min=0).long()] * 2.0, torch.zeros((), dtype=torch.float64, device="cuda")) + B
    has = labels >= 0
    total = torch.nn.functional.cross_entropy((rows @ T.T)[has], labels[has].long(), reduction="sum") / n
    total.backward()
    want = math.sqrt(float((T.grad ** 2).sum() + (B.grad ** 2).sum()))
    f = min(1.0, 0.01 / (want + 1e-6))
    assert f < 1.0
    assert abs(float(loss.double().sum()) / n - float(total.detach())) <= 1e-5 * float(total.detach())
    assert abs(float(norm) - want) <= 1e-5 * want
    for got, ref in ((dtable, T.grad * f), (dbias, B.grad * f)):
        assert float((got.double() - ref).abs().max()) <= 1e-5 * float(ref.abs().max())
    want_x = softmax_reference(x, table, labels, None, 1.0 / n)["dx"]
    assert ((dx.double() - want_x[0]).abs() <= want_x[1]).all()
