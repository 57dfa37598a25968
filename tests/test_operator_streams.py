"""The operators' keyword ``stream`` with the other arguments by place and by name: no GPU is needed, the stream is a stand-in."""
import contextlib

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def operator(monkeypatch):
    from paper_1909_04885_b200 import binding
    current = []

    @contextlib.contextmanager
    def use(stream):
        current.append(stream)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda stream, device: (stream, device))
    monkeypatch.setattr(torch.cuda, "stream", use)

    @binding._operator
    def f(first, second=0, out=None):
        return (list(first) if not isinstance(first, torch.Tensor) else first), second, list(current)

    return f


def test_by_place_and_by_name(operator):
    t = torch.zeros(3)
    for args, kw in (((t, 5), {}), ((t,), {"second": 5}), ((), {"first": t, "second": 5}), ((), {"second": 5, "first": t})):
        assert operator(*args, **kw) == (t, 5, [])
        assert operator(*args, stream=77, **kw) == (t, 5, [(77, t.device)])


def test_several_tensors_by_place_and_by_name(operator):
    a, b = torch.zeros(3), torch.ones(2)
    for make in (lambda: [a, b], lambda: (a, b), lambda: iter([a, b])):
        for args, kw in (((make(),), {}), ((), {"first": make()})):
            assert operator(*args, stream=77, **kw) == ([a, b], 0, [(77, a.device)])
    assert operator([], stream=77) == operator(first=[], stream=77) == ([], 0, [])


def test_a_missing_argument_is_named(operator):
    with pytest.raises(TypeError, match="first"):
        operator(stream=77)
    with pytest.raises(TypeError, match="first"):
        operator(second=3, stream=77)


def test_first_arguments_of_the_operators():
    import inspect

    from paper_1909_04885_b200 import binding
    for name, first in (("softmax_loss", "x"), ("softmax_loss_grad", "x"), ("embedding", "table"), ("embedding_grad", "ids"), ("clip_gradients", "tensors")):
        assert next(iter(inspect.signature(getattr(binding, name)).parameters)) == first
