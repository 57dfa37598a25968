"""Every operator on a stream of the caller's, all arguments by name, on the GPU."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from operator_util import inputs  # noqa: E402


def test_all_arguments_by_name_on_a_stream():
    from paper_1909_04885_b200 import binding, build
    build.build()
    x, w, labels, weights = inputs(60, 90, 40, torch.bfloat16)
    ids = labels % 60
    calls = [lambda **k: binding.softmax_loss(x=x, w=w, labels=labels, **k),
             lambda **k: binding.softmax_loss_grad(x=x, w=w, labels=labels, weights=weights, scale=0.5, **k),
             lambda **k: [binding.embedding(table=x, ids=ids, scale=2.0, **k)],
             lambda **k: [binding.embedding_grad(ids=ids, grad=x, rows=60, **k)],
             lambda **k: [binding.clip_gradients(tensors=[x, w], max_norm=float("inf"), **k)]]
    side = torch.cuda.Stream()
    for f in calls:
        want = f()
        torch.cuda.synchronize()
        got = f(stream=side.cuda_stream)
        side.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(got, want))
