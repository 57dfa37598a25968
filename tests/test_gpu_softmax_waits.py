"""Failure detection in the softmax products without a fault: the copies of some tiles are left out (a test aid, read once per
process, so these run in processes of their own), the waits for them run out within a short limit, every role returns, and the
device goes on."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys, time
sys.path[:0] = [%r, %r]
import torch
from paper_1909_04885_b200 import binding as ops
from operator_util import inputs

def run(n, v, d, dtype, grad, without=0.0):
    x, w, labels, weights = inputs(n, v, d, dtype, without=without)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    out = ops.softmax_loss_grad(x, w, labels, weights=weights, status=status) if grad else ops.softmax_loss(x, w, labels, status=status)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - t0
    assert float(torch.ones(1000, device="cuda").sum()) == 1000.0
    return out, int(status), labels, seconds

%s
print("done")
"""

# single CTAs and pairs, one accumulator and chunks, tiles of 128 and 256 classes, more tiles than CTAs; two tiles at least
SIZES = [(1, 700, 64), (100, 40000, 64), (300, 700, 64), (300, 100, 64), (300, 700, 1100), (2500, 9000, 96)]


def in_a_process(code, tile):
    r = subprocess.run([sys.executable, "-c", CODE % (ROOT, os.path.join(ROOT, "tests"), code)], cwd=ROOT, capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, CHICLE_TEST_DROP_COPIES=str(tile)) if tile is not None else os.environ)
    assert r.returncode == 0 and "done" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


@pytest.mark.parametrize("tile", [0, 1])
def test_copies_that_never_come_end_in_a_status(tile):
    """A launch's waits take 20 M clocks (10 to 20 ms) where they begin, what is in flight as much again at most: of the three products
    of a call, and with the process's own first launches, well under two seconds."""
    in_a_process("""
run(8, 9, 16, torch.bfloat16, True)  # (what a first call loads)
for n, v, d in %r:
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        for grad in (False, True):
            out, status, labels, seconds = run(n, v, d, dtype, grad)
            assert status == ops.STATUS_TIMEOUT, (n, v, d, dtype, grad, status)
            assert seconds < 2.0, (n, v, d, dtype, grad, seconds)
""" % (SIZES,), tile)


def test_without_the_aid_nothing_runs_out():
    in_a_process("""
for n, v, d in %r:
    for grad in (False, True):
        out, status, labels, seconds = run(n, v, d, torch.bfloat16, grad)
        assert status == 0 and all(torch.isfinite(t).all() for t in out)
""" % (SIZES,), None)


@pytest.mark.parametrize("tile", [0, 1, 5])
def test_what_was_not_computed_is_nan(tile):
    """Without a status word, too: a result is NaN or within its bound, rows without a label are 0, and where no tile has its
    operands everything else is NaN."""
    in_a_process("""
from operator_util import softmax_reference
for n, v, d in %r + [(500, 3000, 600)]:
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        x, w, labels, weights = inputs(n, v, d, dtype, without=0.2 if n > 1 else 0.0)
        want = softmax_reference(x, w, labels, weights, 0.5)
        has = labels >= 0
        for f in (lambda: ops.softmax_loss(x, w, labels), lambda: ops.softmax_loss_grad(x, w, labels, weights=weights, scale=0.5)):
            out = dict(zip(("loss", "lse", "dx", "dw"), f()))
            for name, t in out.items():
                ref, off = want[name]
                wrong = torch.isnan(t)
                assert (wrong | ((t.double() - ref).abs() <= off)).all(), (name, n, v, d, dtype)
                if name != "dw":
                    assert not t[~has].any(), (name, n, v, d, dtype)
                if %d == 0:
                    assert (wrong if name == "dw" else wrong[has]).all(), (name, n, v, d, dtype)
            assert torch.isnan(out["loss"]).any() or %d > 1, (n, v, d, dtype)
""" % (SIZES, tile, tile), tile)
