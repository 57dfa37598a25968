"""The widest rows that the operators take (65536 columns), on the GPU. Bounds: operator_util, and of sums by id STEP per term."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import HALF, STEP, TYPES, check, inputs, softmax_reference  # noqa: E402

NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", [(5, 7, 65536), (140, 300, 65535)])
def test_softmax(ops, n, v, d, dtype):
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.1)
    want = softmax_reference(x, w, labels, weights, 0.25)
    for name, t in zip(("loss", "lse"), ops.softmax_loss(x, w, labels)):
        check(t, want[name], name)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.25)):
        check(t, want[name], name)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,d", [(40, 65536), (5000, 65535)])
def test_lookup_and_its_gradient(ops, n, d, dtype):
    v = 30
    table = torch.randn(v, d, device="cuda").to(dtype)
    ids = torch.randint(-1, v, (n,), device="cuda", dtype=torch.int32)
    out = ops.embedding(table, ids, scale=1.5)
    has = ids >= 0
    assert torch.equal(out[has], (table[ids[has].long()].float() * 1.5).to(dtype)) and not out[~has].any()
    got = ops.embedding_grad(ids, out, v)
    for k in range(v):
        terms = out[ids == k].double()
        want = terms.sum(0)
        off = (len(terms) + 2) * STEP * terms.abs().sum(0)
        assert ((got[k].double() - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all()


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
def test_one_column_and_tables_without_rows(ops, dtype):
    x, w, labels, weights = inputs(300, 5, 1, dtype)
    want = softmax_reference(x, w, labels, weights, 1.0)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights)):
        check(t, want[name], name)
    ids = torch.full((70,), -1, device="cuda", dtype=torch.int32)
    ids[3] = 4
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert not ops.embedding(w[:0], ids, status=status).any() and int(status) == ops.STATUS_BAD_ID
    assert ops.embedding_grad(ids, x[:70], 0).shape == (0, 1)
    assert ops.embedding_grad(ids.repeat(100), x[:70].repeat(100, 1), 0).shape == (0, 1)
