"""What the operators without a handle refuse, at the C ABI: no GPU is needed, and none is touched (the addresses are made up)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_1909_04885_b200 import binding, build
    build.build()
    binding.load()
    return binding


A = 1 << 20  # an address like one on a device


def dense(b, rows, cols, type=1, ld=None, data=A):
    return b.Dense(type, rows, cols, cols if ld is None else ld, data)


def call(b, name, *args):
    buf = C.create_string_buffer(256)
    args = [C.byref(a) if isinstance(a, C.Structure) else a for a in args]
    st = getattr(b.load(), name)(0, None, *args, buf, 256)
    return st, buf.value.decode()


def size_of(b, name, *args):
    need = C.c_size_t(12345)
    st = getattr(b.load(), name)(*[C.byref(a) if isinstance(a, C.Structure) else a for a in args], C.byref(need))
    return st, need.value


def test_softmax_workspace_sizes(b):
    x, w = dense(b, 100, 64), dense(b, 1000, 64)
    st, loss = size_of(b, "chicle_softmax_workspace", x, w, 0)
    st2, grad = size_of(b, "chicle_softmax_workspace", x, w, 1)
    assert st == st2 == 0 and 0 < loss < grad and loss % 256 == grad % 256 == 0
    # rows that the bulk copies do not take are copied: more workspace
    assert size_of(b, "chicle_softmax_workspace", dense(b, 100, 64, ld=65), w, 0)[1] > loss
    # the logits are held for a bounded number of rows at a time
    many = [size_of(b, "chicle_softmax_workspace", dense(b, n, 64), dense(b, 131072, 64), 1)[1] for n in (1 << 14, 1 << 16)]
    assert many[1] - many[0] < 1.2 * ((1 << 16) - (1 << 14)) * 64 * 2 + (1 << 26)
    st, kept = size_of(b, "chicle_softmax_workspace", dense(b, 4, 8), dense(b, 4, 9), 1)
    assert st == b.ERR_INVALID_ARG and kept == 12345


@pytest.mark.parametrize("x,w,word", [
    (dict(rows=4, cols=8, type=3), dict(rows=5, cols=8), "type"),
    (dict(rows=4, cols=8, type=0), dict(rows=5, cols=8), "type"),
    (dict(rows=4, cols=8), dict(rows=5, cols=9), "columns"),
    (dict(rows=4, cols=8, ld=7), dict(rows=5, cols=8), "ld"),
    (dict(rows=4, cols=0), dict(rows=5, cols=0), "cols"),
    (dict(rows=-1, cols=8), dict(rows=5, cols=8), "rows"),
    (dict(rows=4, cols=8), dict(rows=0, cols=8), "class"),
    (dict(rows=4, cols=8, data=None), dict(rows=5, cols=8), "NULL"),
    (dict(rows=4, cols=8, data=A + 1), dict(rows=5, cols=8), "aligned"),
    (dict(rows=4, cols=70000), dict(rows=5, cols=70000), "65536"),
    (dict(rows=2 ** 31 - 4096, cols=8), dict(rows=5, cols=8), "2^31"),
    (dict(rows=4, cols=8, ld=2 ** 39), dict(rows=5, cols=8), "ld"),
])
def test_softmax_refuses_matrices(b, x, w, word):
    st, text = call(b, "chicle_softmax_loss", dense(b, **x), dense(b, **w), A, A, A, A, 1 << 40, None)
    assert st == b.ERR_INVALID_ARG and word in text
    assert size_of(b, "chicle_softmax_workspace", dense(b, **x), dense(b, **w), 0)[0] == b.ERR_INVALID_ARG


def test_softmax_refuses_the_rest(b):
    x, w = dense(b, 4, 8), dense(b, 5, 8, data=A + 4096)
    dx, dw = dense(b, 4, 8, data=A + 8192), dense(b, 5, 8, data=A + 12288)
    need = size_of(b, "chicle_softmax_workspace", x, w, 1)[1]
    ws = A + (1 << 16)

    def grad(x=x, w=w, labels=A, weights=None, scale=1.0, loss=A, lse=A, dx=dx, dw=dw, ws=ws, size=need):
        return call(b, "chicle_softmax_loss_grad", x, w, labels, weights, scale, loss, lse, dx, dw, ws, size, None)

    for kw, word in ((dict(labels=None), "labels"), (dict(loss=None), "loss"), (dict(lse=None), "lse"), (dict(size=need - 1), "workspace"),
                     (dict(ws=None), "workspace"), (dict(ws=ws + 16), "aligned"), (dict(scale=float("inf")), "scale"),
                     (dict(dx=dense(b, 3, 8, data=A + 8192)), "dX"), (dict(dw=dense(b, 5, 8, type=2, data=A + 12288)), "dW"),
                     (dict(dx=dense(b, 4, 8, data=A)), "overlap"), (dict(dw=dense(b, 5, 8, data=A + 4096 + 64)), "overlap"),
                     (dict(dw=dense(b, 5, 8, data=A + 8192 + 32)), "overlap"), (dict(dw=None), "NULL")):
        st, text = grad(**kw)
        assert st == b.ERR_INVALID_ARG and word in text, (kw, text)
    st, text = call(b, "chicle_softmax_loss", x, w, None, A, A, ws, need, None)
    assert st == b.ERR_INVALID_ARG and "labels" in text


def test_embedding_refuses(b):
    t, o = dense(b, 10, 8), dense(b, 4, 8, data=A + 4096)
    need = size_of(b, "chicle_embedding_grad_workspace", 4, 10, 8)[1]
    assert need > 0 and size_of(b, "chicle_embedding_grad_workspace", 0, 10, 8) == (0, 0)
    for args in ((-1, 10, 8), (4, -1, 8), (4, 10, 0), (2 ** 31, 10, 8), (4, 2 ** 31, 8), (4, 10, 70000)):
        assert size_of(b, "chicle_embedding_grad_workspace", *args) == (b.ERR_INVALID_ARG, 12345)
    for args, word in (((t, None, 1.0, o, None), "ids"), ((t, A, float("nan"), o, None), "scale"),
                       ((t, A, 1.0, dense(b, 4, 7, data=A + 4096), None), "columns"), ((t, A, 1.0, dense(b, 4, 8, type=0, data=A + 4096), None), "type"),
                       ((t, A, 1.0, dense(b, 4, 8, data=A + 32), None), "overlap")):
        st, text = call(b, "chicle_embedding", *args)
        assert st == b.ERR_INVALID_ARG and word in text
    ws = A + (1 << 16)
    for args, word in (((None, o, 1.0, 0, t, ws, need, None), "ids"), ((A, o, 1.0, 0, t, ws, need - 1, None), "workspace"),
                       ((A, o, 1.0, 0, t, ws + 8, need, None), "aligned"), ((A, o, 1.0, 0, dense(b, 10, 8, data=A + 4096), ws, need, None), "overlap")):
        st, text = call(b, "chicle_embedding_grad", *args)
        assert st == b.ERR_INVALID_ARG and word in text


def test_clipping_refuses(b):
    class Tensor(C.Structure):
        _fields_ = [("type", C.c_int), ("n", C.c_int64), ("inp", C.c_void_p), ("out", C.c_void_p)]

    def clip(tensors, max_norm=1.0, norm=A, ws=A, size=b.CLIP_WORKSPACE, count=None):
        table = (Tensor * max(1, len(tensors)))(*[Tensor(*t) for t in tensors])
        return call(b, "chicle_clip_gradients", len(tensors) if count is None else count, C.cast(table, C.c_void_p), max_norm, norm, ws, size)

    assert C.sizeof(Tensor) == 32
    good = (1, 100, A, A)
    for kw, word in ((dict(max_norm=-1.0), "max_norm"), (dict(max_norm=float("nan")), "max_norm"), (dict(norm=None), "norm"),
                     (dict(size=b.CLIP_WORKSPACE - 1), "workspace"), (dict(ws=A + 8), "aligned"), (dict(count=-1), "count")):
        st, text = clip([good], **kw)
        assert st == b.ERR_INVALID_ARG and word in text
    for tensors, word in (([(3, 100, A, A)], "type"), ([(1, -1, A, A)], "length"), ([(1, 2 ** 41, A, A)], "length"), ([(1, 100, None, None)], "NULL"),
                          ([(0, 100, A + 2, A + 2)], "aligned"), ([good, good], "out"), ([(1, 100, A, A + 100)], "out"),
                          ([good, (1, 10, A + 4096, A + 100)], "out"), ([(1, 100, A, A + 8192), (1, 100, A + 4096, A + 8192 + 198)], "out"),
                          ([(1, 100, A, A + 8192), (1, 100, A + 8192, None)], "out")):
        st, text = clip(tensors)
        assert st == b.ERR_INVALID_ARG and word in text, (tensors, text)


def test_without_a_gpu_they_fail_loudly(b):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    x, w = dense(b, 4, 8), dense(b, 5, 8, data=A + 4096)
    need = size_of(b, "chicle_softmax_workspace", x, w, 0)[1]
    st, text = call(b, "chicle_softmax_loss", x, w, A, A, A, A + (1 << 16), need, None)
    assert st == b.ERR_CUDA and text
    with pytest.raises(ValueError):
        b.softmax_loss(torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        b.clip_gradients([torch.zeros(4)], 1.0)
