"""Embedding lookup and its gradient against 64 bits, on the GPU."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import HALF, STEP, TYPES  # noqa: E402

NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


def some_ids(n, v, seed=0, kind="mixed"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "mixed":  # one id has a third of the entries, some entries have none
        r = torch.rand(n, generator=g, device="cuda")
        ids = torch.where(r < 0.33, torch.full_like(ids, v // 2), ids)
        ids = torch.where(r > 0.9, torch.full_like(ids, -1), ids)
    elif kind == "one":
        ids.fill_(v - 1)
    elif kind == "none":
        ids.fill_(-7)
    return ids


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (5, 3, 7), (32, 100, 4096), (1000, 50, 33), (40000, 999, 64), (20000, 7, 66), (3, 9, 20000)])
def test_lookup(ops, n, v, d, dtype):
    table = torch.randn(v, d, device="cuda").to(dtype)
    ids = some_ids(n, v)
    want = torch.where((ids >= 0)[:, None], table[ids.clamp(min=0).long()].float() * 1.75, torch.zeros((), device="cuda")).to(dtype)
    got = ops.embedding(table, ids, scale=1.75)
    assert torch.equal(got, want)  # one product in fp32, one rounding: the same bits


def test_lookup_of_strided_rows(ops):
    wide = torch.randn(50, 101, device="cuda")
    ids = some_ids(300, 50)
    out = torch.full((300, 70), 7.0, device="cuda")
    ops.embedding(wide[:, 3:67], ids, scale=0.5, out=out[:, 1:65])
    want = torch.where((ids >= 0)[:, None], wide[:, 3:67][ids.clamp(min=0).long()] * 0.5, torch.zeros((), device="cuda"))
    assert torch.equal(out[:, 1:65], want)
    assert (out[:, 0] == 7).all() and (out[:, 65:] == 7).all()


def check_grad(ops, ids, grad, v, scale, into=None):
    dt = grad.dtype
    has = (ids >= 0) & (ids < v)
    at = ids[has].long()
    terms = grad[has].double()
    ref = torch.zeros(v, grad.shape[1], dtype=torch.float64, device="cuda").index_add_(0, at, terms) * scale
    mag = torch.zeros_like(ref).index_add_(0, at, terms.abs()) * abs(scale)
    count = torch.bincount(at, minlength=v).double()[:, None]
    if into is None:
        got = ops.embedding_grad(ids, grad, v, scale=scale)
        base = torch.zeros_like(ref)
    else:
        base = into.double()
        got = ops.embedding_grad(ids, grad, v, scale=scale, out=into, accumulate=True)
        assert got is into
    want = ref + base
    # count terms added in fp32, the product with the scale, the sum with what was there, one rounding
    off = (count + 2) * STEP * mag + STEP * want.abs()
    off = off + HALF[dt] * (want.abs() + off) + torch.finfo(dt).smallest_normal * 2 * HALF[dt]
    off = torch.where(count > 0, off, torch.zeros_like(off))  # rows without an id: exactly 0, or what was there
    err = (got.double() - want).abs()
    assert (err <= off).all(), float((err / off.clamp(min=1e-300)).max())
    return got


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d,kind", [
    (1, 1, 1, "flat"), (1, 5, 16, "none"), (7, 3, 5, "mixed"), (8, 4, 8, "one"), (100, 1000, 64, "mixed"), (4096, 300, 40, "mixed"),
    (4097, 300, 40, "mixed"), (8192, 5000, 20, "mixed"), (8193, 5000, 20, "mixed"), (5000, 70000, 33, "flat"), (9000, 17, 1024, "mixed"), (20000, 1, 16, "one"), (30000, 3000000, 8, "mixed"),
    (140000, 1200, 20, "mixed"), (6000, 900, 2100, "mixed"), (9001, 900, 2100, "mixed"), (8500, 17, 1024, "one"), (10000, 40, 12, "none"), (300000, 1023, 4, "mixed"), (300000, 1024, 4, "mixed")])
def test_gradient(ops, n, v, d, kind, dtype):
    g = torch.Generator(device="cuda").manual_seed(5)
    grad = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    ids = some_ids(n, v, kind=kind)
    a = check_grad(ops, ids, grad, v, 0.7)
    assert torch.equal(a, ops.embedding_grad(ids, grad, v, scale=0.7))  # the same bits again


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n", [300, 9000])
def test_gradient_added_to_what_is_there(ops, n, dtype):
    v, d = 200, 72
    grad = torch.randn(n, d, device="cuda").to(dtype)
    ids = some_ids(n, v // 2)  # half of the rows get nothing
    into = torch.randn(v, d, device="cuda").to(dtype)
    into[v // 2:] = float("nan")  # and are not looked at
    keep = into.clone()
    into[v // 2:] = 1.0
    check_grad(ops, ids, grad, v, -1.25, into=into)
    keep2 = keep.clone()
    ops.embedding_grad(ids, grad, v, out=keep2, accumulate=True)
    assert torch.isnan(keep2[v // 2:]).all() and not torch.isnan(keep2[:v // 2]).any()


@pytest.mark.parametrize("n", [200, 8000, 9000])
def test_gradient_of_strided_rows(ops, n):
    wide = torch.randn(n, 90, device="cuda", dtype=torch.bfloat16)
    ids = some_ids(n, 40)
    out = torch.full((40, 80), 3.0, device="cuda", dtype=torch.bfloat16)
    ops.embedding_grad(ids, wide[:, 7:71], 40, out=out[:, 5:69])
    assert torch.equal(out[:, 5:69], ops.embedding_grad(ids, wide[:, 7:71].contiguous(), 40))
    assert (out[:, :5] == 3).all() and (out[:, 69:] == 3).all()


@pytest.mark.parametrize("n", [50, 6000, 9000])
def test_ids_beyond_the_last_row(ops, n):
    ids = some_ids(n, 30, kind="flat")
    bad, without = ids.clone(), ids.clone()
    bad[[3, 20]] = torch.tensor([30, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    without[[3, 20]] = -1
    table, grad = torch.randn(30, 16, device="cuda"), torch.randn(n, 16, device="cuda")
    for f in (lambda i, s: ops.embedding(table, i, status=s), lambda i, s: ops.embedding_grad(i, grad, 30, status=s)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        assert torch.equal(f(bad, status), f(without, None))
        assert int(status) == ops.STATUS_BAD_ID
        status.zero_()
        f(without, status)
        assert int(status) == 0


def test_masked_rows_hold_nan(ops):
    ids = some_ids(500, 20)
    grad = torch.randn(500, 24, device="cuda")
    grad[ids < 0] = float("nan")
    assert torch.isfinite(ops.embedding_grad(ids, grad, 20)).all()


def test_no_ids(ops):
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ops.embedding(torch.randn(4, 8, device="cuda"), none).shape == (0, 8)
    grad = torch.empty(0, 8, device="cuda")
    assert not ops.embedding_grad(none, grad, 4).any()
    into = torch.ones(4, 8, device="cuda")
    ops.embedding_grad(none, grad, 4, out=into, accumulate=True)
    assert (into == 1).all()


@pytest.mark.parametrize("n", [1000, 9000])
def test_captured(ops, n):
    ids, grad, table = some_ids(n, 300), torch.randn(n, 48, device="cuda"), torch.randn(300, 48, device="cuda")
    ops.embedding_grad(ids, grad, 300)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, back = ops.embedding(table, ids, scale=2.0), ops.embedding_grad(ids, grad, 300, scale=2.0)
    ids.copy_(some_ids(n, 300, seed=1))
    grad.copy_(torch.randn(n, 48, device="cuda"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ops.embedding(table, ids, scale=2.0))
    assert torch.equal(back, ops.embedding_grad(ids, grad, 300, scale=2.0))


def test_a_table_beyond_32_bit_offsets(ops):
    """2.2 G elements: rows in front of and behind element 2^31, and behind byte 2^32."""
    v, d = 1_100_000, 2048
    table = torch.empty(v, d, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1, 2 ** 20 - 1, 2 ** 20, 2 ** 20 + 1, 2 ** 21 // 2 + 5000, v - 2, v - 1], device="cuda")
    table[rows] = torch.randn(8, d, device="cuda").bfloat16()
    ids = rows.int().repeat(700)
    assert torch.equal(ops.embedding(table, ids), table[rows].repeat(700, 1))
    grad = torch.randn(len(ids), d, device="cuda").bfloat16()
    for n in (64, 5600):  # sorted by counting, and by radix passes
        table.fill_(1.0)
        got = ops.embedding_grad(ids[:n], grad[:n], v, out=table)
        want = grad[:n].double().view(-1, 8, d).sum(0)
        off = n * STEP * grad[:n].double().abs().view(-1, 8, d).sum(0)
        assert ((got[rows].double() - want).abs() <= off + HALF[torch.bfloat16] * (want.abs() + off)).all()
        got[rows] = 0
        assert not got.any()


def test_refusals(ops):
    table, ids, grad = torch.randn(6, 8, device="cuda"), some_ids(4, 6), torch.randn(4, 8, device="cuda")
    for f in (lambda: ops.embedding(table.T, ids), lambda: ops.embedding(table, ids.long()), lambda: ops.embedding(table.cpu(), ids),
              lambda: ops.embedding(table, ids, out=table[:4]), lambda: ops.embedding(table, ids, scale=float("inf")),
              lambda: ops.embedding(table, ids, out=torch.empty(3, 8, device="cuda")),
              lambda: ops.embedding_grad(ids, grad[:3], 6), lambda: ops.embedding_grad(ids, grad, 6, accumulate=True),
              lambda: ops.embedding_grad(ids, grad, 6, out=torch.empty(6, 8, device="cuda", dtype=torch.float16)),
              lambda: ops.embedding_grad(ids, grad, -1)):
        with pytest.raises((ValueError, RuntimeError, ops.ChicleError)):
            f()
