"""Plain 64-bit forms of the operators of a softmax model, and how far the kernels' results may be from them.

The bounds are worst cases of what the kernels do, element by element: a rounding to a type is off by half a step
(HALF), a sum of k terms in fp32 by k STEP times the sum of the terms' magnitudes (STEP = 2^-23: the tensor cores may cut off
instead of rounding), and what that does to a function of the sum.
"""
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
STEP = 2.0 ** -23
TYPES = [torch.float32, torch.bfloat16, torch.float16]


FEW = 32  # rows up to which 16-bit P is held in two planes


def softmax_reference(x, w, labels, weights=None, scale=1.0):
    """Everything in 64 bits: loss, lse, dx, dw and, for each, the largest error allowed (element by element)."""
    dt = x.dtype
    X, W = x.double(), w.double()
    n, d = X.shape
    v = W.shape[0]
    has = (labels >= 0) & (labels < v)
    X = torch.where(has[:, None], X, torch.zeros_like(X))  # what a row without a label holds has no effect
    at = torch.where(has, labels, torch.zeros_like(labels)).long()
    logits = X @ W.T
    lse = torch.logsumexp(logits, 1)
    loss = lse - logits.gather(1, at[:, None])[:, 0]
    soft = (logits - lse[:, None]).exp()
    g = (torch.ones(n, device=x.device) if weights is None else weights).double() * scale
    g = torch.where(has, g, torch.zeros_like(g))
    p = soft.clone()
    p[torch.arange(n, device=x.device), at] -= 1.0
    p *= g[:, None]
    zero = torch.zeros_like(lse)
    # a logit: a sum of d products. Single precision: of 3 d products of planes; a plane pair is off by 2^-22 (2 STEP) of an
    # element or 2^-39 of the largest one, either factor, and the product left out is 2^-22 of a term: 8 STEP of it in all
    single = dt == torch.float32
    terms = 3 * d + 8 if single else d
    off = (terms * STEP * (X.abs() @ W.abs().T)).amax(1)
    if single:
        off = off + 2.0 ** -38 * (X.abs().max() * W.abs().sum(1).max() + W.abs().max() * X.abs().sum(1))
    # lse and loss: the logits' error, exponentials, their sum and the logarithm, the largest logit's rounding when added
    off_lse = torch.where(has, off + (v / 16 + 32) * STEP + 2 * STEP * (lse.abs() + logits.abs().amax(1)), zero)
    off_loss = torch.where(has, 2 * off + (v / 16 + 32) * STEP + 4 * STEP * (loss.abs() + logits.abs().amax(1)), zero)
    # an entry of P: of exp(logit - lse) the two errors and the exponentials' (16 steps); its storage in between (fp16, 2^-11,
    # and of small ones 2^-40 of the largest) and its rounding; fp16 and its planes: of the lifted value, which may be subnormal
    gs = g.abs()[:, None]
    rel = (2 * (off + off_lse) + 16 * STEP)[:, None]
    planes = single or n <= FEW  # (two planes: the rounding of what the first one is off by; bf16 2^-16)
    off_p = soft * gs * rel + p.abs() * (4 * STEP if single else HALF[dt] ** 2 + 4 * STEP if planes else HALF[dt])
    if not single:
        off_p = off_p + soft * gs * 2.0 ** -11 + gs * 2.0 ** -40
    if dt != torch.bfloat16:
        off_p = off_p + float(gs.max()) * 2.0 ** -37
    Wa, Xa = W.abs(), X.abs()
    pa = p.abs() + off_p
    k = 3 if single else 2 if planes else 1
    tiny = torch.finfo(dt).smallest_normal * 2 * HALF[dt]
    dx, dw = p @ W, p.T @ X
    off_dx = off_p @ Wa + (k * v + 8) * STEP * (pa @ Wa) + HALF[dt] * dx.abs() * (1 + 2 * HALF[dt]) + tiny
    off_dw = off_p.T @ Xa + (k * (n + 64) + 8) * STEP * (pa.T @ Xa) + HALF[dt] * dw.abs() * (1 + 2 * HALF[dt]) + tiny
    if single:
        off_dx = off_dx + 2.0 ** -38 * Wa.max() * pa.sum(1, keepdim=True)
        off_dw = off_dw + 2.0 ** -38 * Xa.max() * pa.sum(0)[:, None]
    off_dx = off_dx + HALF[dt] * (off_p @ Wa)  # (the rounding is of the computed value)
    off_dw = off_dw + HALF[dt] * (off_p.T @ Xa)
    off_dx = torch.where(has[:, None], off_dx, torch.zeros_like(off_dx))
    return {"loss": (torch.where(has, loss, zero), off_loss), "lse": (torch.where(has, lse, zero), off_lse), "dx": (dx, off_dx),
            "dw": (dw, off_dw)}


def check(got, want, name):
    ref, off = want
    err = (got.double() - ref).abs()
    bad = ~(err <= off)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g of its bound" % (name, int(bad.sum()), bad.numel(), float((err / off.clamp(min=1e-300)).max()))


def inputs(n, v, d, dtype, seed=0, spread=2.0, without=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    w = (torch.randn(v, d, generator=g, device="cuda") * (spread / d ** 0.5)).to(dtype)
    labels = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    if without:
        labels = torch.where(torch.rand(n, generator=g, device="cuda") < without, torch.full_like(labels, -1), labels)
    weights = torch.rand(n, generator=g, device="cuda") + 0.5
    return x, w, labels, weights
