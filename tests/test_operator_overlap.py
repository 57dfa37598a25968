"""Which matrices the operators take for overlapping, at the C ABI: no GPU is needed, and none is touched (the addresses are made
up, and a scale that is not finite refuses every call that this check lets pass)."""
import ctypes as C
import random

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_1909_04885_b200 import binding, build
    build.build()
    binding.load()
    return binding


A = 1 << 20


def refused_for(b, table, out):
    buf = C.create_string_buffer(256)
    st = b.load().chicle_embedding(0, None, C.byref(table), A, float("nan"), C.byref(out), None, buf, 256)
    assert st == b.ERR_INVALID_ARG
    return "overlap" if b"overlap" in buf.value else "scale" if b"scale" in buf.value else buf.value


def spans(m):
    es = 4 if m.type == 0 else 2
    return {m.data + i * m.ld * es + j for i in range(m.rows) for j in range(m.cols * es)}


def test_against_all_bytes(b):
    rng = random.Random(3)
    seen = {"overlap": 0, "scale": 0}
    for _ in range(20000):
        type, cols = rng.choice([0, 1, 2]), rng.randint(1, 5)
        es = 4 if type == 0 else 2
        ld = cols + rng.randint(0, 9)
        other = ld if rng.random() < 0.7 else cols + rng.randint(0, 9)
        x = b.Dense(type, rng.randint(0, 4), cols, ld, A)
        y = b.Dense(type, rng.randint(0, 4), cols, other, A + es * rng.randint(-60, 60))
        p, q = spans(x), spans(y)
        if x.rows > 1 and y.rows > 1 and ld != other:
            want = not (max(p) < min(q) or max(q) < min(p))
        else:
            want = bool(p & q)
        want = "overlap" if want else "scale"
        assert refused_for(b, x, y) == want and refused_for(b, y, x) == want, (x.type, x.rows, cols, ld, other, y.rows, y.data - A)
        seen[want] += 1
    assert min(seen.values()) > 1000


def test_columns_of_one_buffer(b):
    """Operands and gradients side by side: what the call says next is about the scale."""
    x, w = b.Dense(1, 100, 32, 200, A), b.Dense(1, 50, 32, 200, A + 64)
    dx, dw = b.Dense(1, 100, 32, 200, A + 128), b.Dense(1, 50, 32, 200, A + 192)
    buf = C.create_string_buffer(256)
    for second, word in ((dx, b"scale"), (b.Dense(1, 100, 32, 200, A + 126), b"overlap")):
        st = b.load().chicle_softmax_loss_grad(0, None, C.byref(x), C.byref(w), A, None, float("inf"), A, A, C.byref(second), C.byref(dw), A, 1 << 40,
                                               None, buf, 256)
        assert st == b.ERR_INVALID_ARG and word in buf.value


def test_far_pitches(b):
    """Extents beyond 64 bits."""
    far = b.Dense(1, 2 ** 31 - 5000, 8, 2 ** 38, A)
    assert refused_for(b, far, b.Dense(1, 4, 8, 8, A + 4096)) == "overlap"  # (different pitches: by extent)
    assert refused_for(b, far, b.Dense(1, 4, 8, 2 ** 38, A + 16)) == "scale"
    assert refused_for(b, far, b.Dense(1, 4, 8, 2 ** 38, A + 14)) == "overlap"
    assert refused_for(b, far, b.Dense(1, 1, 8, 8, A + 2 ** 39 * 1000 + 14)) == "overlap"
    assert refused_for(b, far, b.Dense(1, 1, 8, 8, A + 2 ** 39 * 1000 + 16)) == "scale"
