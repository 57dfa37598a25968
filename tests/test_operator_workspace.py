"""How much workspace the gradients of a softmax model ask for, at the C ABI: no GPU is needed."""
import ctypes as C

import pytest

GIB = 1 << 30


@pytest.fixture(scope="module")
def b():
    from paper_1909_04885_b200 import binding, build
    build.build()
    binding.load()
    return binding


def size_of(b, n, v, d, type, grad=1):
    need = C.c_size_t()
    x, w = b.Dense(type, n, d, d, 1 << 20), b.Dense(type, v, d, d, 1 << 40)
    assert b.load().chicle_softmax_workspace(C.byref(x), C.byref(w), grad, C.byref(need)) == 0
    return need.value


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("v", [100, 131072, 1_000_000, 4_000_000, 10_000_000, 20_000_000, 50_000_000, 100_000_000, 1_000_000_000])
@pytest.mark.parametrize("n", [1, 32, 33, 255, 256, 300, 2047, 4096, 100_000])
def test_logits_of_a_piece_are_bounded(b, n, v, type):
    """8 GiB of logits and a 32nd of it for their sums (fp32: a 64th), beside what the matrices' own sizes ask for: X and W laid out
    (fp32: two planes), the fp32 sums of dW, and the pieces' dX."""
    d, line = 8, 64
    planes = 2 if type == 0 else 1
    beside = planes * n * line * 2 + (planes * v * line * 2 if type == 0 else 0) + v * d * 4 + 64 * min(n, 1 << 23) * d * 4
    assert size_of(b, n, v, d, type) <= max(8 * GIB, v * 8) * 33 // 32 + beside + (1 << 20)


def test_sizes_with_room_are_as_they_were(b):
    """Where 2048 rows take less than 8 GiB, pieces are whole tiles: more rows beyond one piece only add their own layout."""
    for type, planes in ((0, 2), (1, 1), (2, 1)):
        a, c = size_of(b, 1 << 14, 131072, 64, type), size_of(b, 1 << 16, 131072, 64, type)
        assert c - a == planes * ((1 << 16) - (1 << 14)) * 64 * 2


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("grad", [0, 1])
def test_no_rows(b, type, grad):
    assert size_of(b, 0, 100, 8, type, grad) >= 0
