"""More rows in one piece than a launch of the elementwise pass takes (65535), few classes, on the GPU. Bounds: operator_util."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import TYPES, check, inputs, softmax_reference  # noqa: E402

NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES.get)
@pytest.mark.parametrize("n,v,d", [(65535, 3, 28), (65536, 10, 28), (140000, 100, 20), (200000, 2, 5)])
def test_rows_beyond_one_launch(n, v, d, dtype):
    from paper_1909_04885_b200 import binding, build
    build.build()
    x, w, labels, weights = inputs(n, v, d, dtype, without=0.1)
    labels[65535 % n], labels[n - 1], labels[n - 3] = 1, 0, v  # (the last but two has a label beyond the last class)
    want = softmax_reference(x, w, labels, weights, 1.0 / n)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for name, t in zip(("loss", "lse", "dx", "dw"), binding.softmax_loss_grad(x, w, labels, weights=weights, scale=1.0 / n, status=status)):
        check(t, want[name], name)
    assert int(status) == binding.STATUS_BAD_ID
    for name, t in zip(("loss", "lse"), binding.softmax_loss(x, w, labels)):
        check(t, want[name], name)
