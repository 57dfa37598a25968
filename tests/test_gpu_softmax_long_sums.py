"""Gradients in 16 bits whose sums have more terms than one accumulator takes (12288 in fp16, 98304 in bf16, half of that where P has
two planes), on the GPU. As many tiles as there are SMs or pairs of them, so that the sums are not cut for the SMs' sake. Bounds:
operator_util."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import check, inputs, softmax_reference  # noqa: E402

NAMES = {torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.fixture(scope="module")
def ops():
    from paper_1909_04885_b200 import binding, build
    build.build()
    return binding


# dX with one slice more than an accumulator takes, and in two whole chunks; dW; P in two planes; tiles of 128 columns; both in bf16
@pytest.mark.parametrize("n,v,d,dtype", [
    (2300, 12289, 2047, torch.float16), (2304, 24576, 2048, torch.float16), (12350, 2300, 2047, torch.float16), (20, 6200, 36000, torch.float16),
    (18900, 12500, 100, torch.float16), (12500, 18900, 128, torch.float16), (2300, 99000, 2047, torch.bfloat16), (99000, 2300, 2047, torch.bfloat16)],
    ids=lambda t: NAMES.get(t, t) if isinstance(t, torch.dtype) else t)
def test_gradients(ops, n, v, d, dtype):
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.1)
    want = softmax_reference(x, w, labels, weights, 1.0)
    for name, t in zip(("loss", "lse", "dx", "dw"), ops.softmax_loss_grad(x, w, labels, weights=weights)):
        check(t, want[name], name)
    again = ops.softmax_loss_grad(x, w, labels, weights=weights)
    # the norms: each rounding half / sqrt(3) in the mean, the result's and P's, and a tenth for the rest (as in the tests of accuracy)
    half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    for name, t in zip(("dx", "dw"), again[2:]):
        ref = want[name][0]
        assert float((t.double() - ref).norm() / ref.norm()) <= 1.1 * 2 ** 0.5 * half / 3 ** 0.5, name


@pytest.mark.parametrize("n,v,d", [(2300, 12400, 2047), (12350, 2300, 2047)])
def test_into_columns_of_a_buffer(ops, n, v, d):
    """Results with an odd pitch at an odd place: the bits of whole rows, and nothing beside them is written."""
    import ctypes as C
    dtype = torch.float16
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.1)
    want = ops.softmax_loss_grad(x, w, labels, weights=weights)
    gx, gw = (torch.full((k, d + 6), 7.0, dtype=dtype, device="cuda") for k in (n, v))
    desc = [ops._dense(t, "a matrix") for t in (x, w, gx[:, 3:3 + d], gw[:, 3:3 + d])]
    need, buf = C.c_size_t(), C.create_string_buffer(256)
    lib = ops.load()
    assert lib.chicle_softmax_workspace(C.byref(desc[0]), C.byref(desc[1]), 1, C.byref(need)) == 0
    ws, out = torch.empty(need.value, dtype=torch.uint8, device="cuda"), torch.empty(2, n, device="cuda")
    st = lib.chicle_softmax_loss_grad(0, torch.cuda.current_stream().cuda_stream, C.byref(desc[0]), C.byref(desc[1]), labels.data_ptr(), weights.data_ptr(),
                                      1.0, out[0].data_ptr(), out[1].data_ptr(), C.byref(desc[2]), C.byref(desc[3]), ws.data_ptr(), need.value, None, buf, 256)
    assert st == 0, buf.value
    for got, ref in ((gx, want[2]), (gw, want[3])):
        assert torch.equal(got[:, 3:3 + d], ref) and (got[:, :3] == 7).all() and (got[:, 3 + d:] == 7).all()
