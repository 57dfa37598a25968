"""Operands and results side by side in the columns of one buffer, on the GPU: the bits of separate buffers, and nothing beside
the results is written."""
import ctypes as C

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import TYPES, inputs  # noqa: E402

NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d,gap", [(150, 333, 72, 8), (150, 333, 33, 3), (20, 90, 64, 0)])
def test_gradients_beside_their_operands(ops, n, v, d, gap, dtype):
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.1)
    want = ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.5)
    step = d + gap
    pool = torch.full((max(n, v), 4 * step), 7.0, dtype=dtype, device="cuda")
    cut = [pool[:k, i * step:i * step + d] for i, k in enumerate((n, v, n, v))]  # x, w, dx, dw
    cut[0].copy_(x)
    cut[1].copy_(w)
    keep = pool.clone()
    desc = [ops._dense(t, "a matrix") for t in cut]
    need = C.c_size_t()
    lib = ops.load()
    assert lib.chicle_softmax_workspace(C.byref(desc[0]), C.byref(desc[1]), 1, C.byref(need)) == 0
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(2, n, device="cuda")
    buf = C.create_string_buffer(256)
    st = lib.chicle_softmax_loss_grad(0, torch.cuda.current_stream().cuda_stream, C.byref(desc[0]), C.byref(desc[1]), labels.data_ptr(), weights.data_ptr(),
                                      0.5, loss.data_ptr(), lse.data_ptr(), C.byref(desc[2]), C.byref(desc[3]), ws.data_ptr(), need.value, None, buf, 256)
    assert st == 0, buf.value
    for s, t in zip((loss, lse, cut[2], cut[3]), want):
        assert torch.equal(s, t)
    keep[:n, 2 * step:2 * step + d] = want[2]
    keep[:v, 3 * step:3 * step + d] = want[3]
    assert torch.equal(pool, keep)


@pytest.mark.parametrize("n", [50, 6000])
def test_vectors_beside_their_table(ops, n):
    v, d = 6000, 24
    table = torch.randn(v, d, device="cuda")
    ids = torch.randint(-1, v, (n,), device="cuda", dtype=torch.int32)
    pool = torch.full((v, 3 * d + 2), 7.0, device="cuda")
    pool[:, :d] = table
    out, back = pool[:n, d + 1:2 * d + 1], pool[:, 2 * d + 1:3 * d + 1]
    ops.embedding(pool[:, :d], ids, scale=3.0, out=out)
    assert torch.equal(out, ops.embedding(table, ids, scale=3.0))
    ops.embedding_grad(ids, out, v, out=back)
    assert torch.equal(back, ops.embedding_grad(ids, out.contiguous(), v))
    assert torch.equal(pool[:, :d], table) and (pool[:, d] == 7).all() and (pool[:, 3 * d + 1:] == 7).all() and (pool[n:, d + 1:2 * d + 1] == 7).all()
