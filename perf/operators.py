"""The operators around a softmax model with a vector per id, as measurable cases.

A model over hashed or tokenised ids has a table with one vector per id at its input and a linear map to the classes
(or the vocabulary) at its output. A training step looks vectors up (`embedding`), takes the softmax cross entropy of
the linear map and its gradients (`softmax_loss_grad`), sums the gradient of the looked-up vectors by id
(`embedding_grad`) and clips all gradients by their common norm (`clip_gradients`); an evaluation, or the score of
one next id, takes the loss alone (`softmax_loss`).

`run` makes these calls of the package where `own` is true, and computes the same with elementary torch operations
where it is not. All inputs are synthetic and drawn from the seed on the GPU.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
LARGEST = 8192 * 131072 * 4096  # n * v * d of the largest listed loss


# ------------------------------------------------------------------------------------------------ cases
def _loss(name, op, n, v, d, dtype, ignored=0.0):
    return {"name": name, "op": op, "n": n, "v": v, "d": d, "dtype": dtype, "ignored": ignored}


def _ids(name, op, n, v, d, dtype, ignored=0.0):
    return {"name": name, "op": op, "n": n, "v": v, "d": d, "dtype": dtype, "ignored": ignored}


def _clip(name, layers, d, v, dtype, factor):
    return {"name": name, "op": "clip", "layers": layers, "d": d, "v": v, "dtype": dtype, "factor": factor}


def listed():
    return [
        # the score of one next id against the whole vocabulary: the weights are read once, little else
        _loss("loss_one_row", "loss", 1, 131072, 4096, "bf16"),
        # an evaluation pass over a batch, with rows that have no label
        _loss("loss_eval", "loss", 4096, 100000, 2048, "bf16", 0.1),
        # classes of a small dense table, single precision: the smallest training step, launches and latency
        _loss("grad_classes_fp32", "grad", 10000, 1000, 100, "fp32"),
        # odd sizes throughout in half precision
        _loss("grad_odd_fp16", "grad", 1777, 50001, 1000, "fp16", 0.1),
        # a training step of a mid-size model in single precision
        _loss("grad_fp32", "grad", 2048, 32768, 1024, "fp32"),
        # a training step of a large model
        _loss("grad_train", "grad", 8192, 131072, 4096, "bf16", 0.05),
        # the vectors of one id per request of a small batch: latency
        _ids("embedding_decode", "embedding", 32, 131072, 4096, "bf16"),
        # 8192 hashed rows of 39 ids each, over a million ids
        _ids("embedding_hashed", "embedding", 319488, 1000000, 128, "fp32"),
        # the gradient of a training step's tokens, with padding
        _ids("embedding_grad_tokens", "embedding_grad", 16384, 131072, 4096, "bf16", 0.05),
        # the gradient of the hashed rows: many ids that come once, a few that come thousands of times
        _ids("embedding_grad_hashed", "embedding_grad", 319488, 1000000, 64, "fp32"),
        # a small model's gradients: launches and latency
        _clip("clip_small", 12, 64, 1000, "fp32", 0.4),
        # a large model's gradients
        _clip("clip_large", 24, 2048, 131072, "bf16", 0.3),
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["loss", "grad", "grad", "embedding", "embedding_grad", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("loss", "grad"):
        while True:
            n, v, d = _log(rng, 1, 16384), _log(rng, 2, 200000), _log(rng, 16, 4096)
            if rng.random() < 0.5:  # widths are mostly even ones
                d = max(16, d // 64 * 64)
            if n * v * d <= LARGEST and n * v <= 8192 * 131072:
                return _loss("drawn", op, n, v, d, dtype, rng.choice([0.0, 0.1]))
    if op in ("embedding", "embedding_grad"):
        while True:
            n, v, d = _log(rng, 1, 400000), _log(rng, 2, 1000000), _log(rng, 16, 4096)
            if rng.random() < 0.5:
                d = max(16, d // 64 * 64)
            if max(n, v) * d <= 131072 * 4096:
                return _ids("drawn", op, n, v, d, dtype, rng.choice([0.0, 0.1]))
    return _clip("drawn", rng.randint(1, 12 if dtype == "fp32" else 24), _log(rng, 32, 2048), _log(rng, 100, 131072), dtype, rng.choice([0.1, 0.9, 2.0]))


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _skewed(n, v, g):
    """n ids of 0 .. v-1: frequencies like one over the rank, ranks scattered over the ids."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    rank = torch.exp(u * math.log(v + 1)).long().sub_(1).clamp_(0, v - 1)
    return torch.randperm(v, generator=g, device=DEV)[rank].int()


def _without(ids, share, g):
    """Marks a share of the ids as having none (-1)."""
    if share:
        ids = torch.where(torch.rand(ids.shape, generator=g, device=DEV) < share, torch.full_like(ids, -1), ids)
    return ids


def _clip_sizes(case):
    d = case["d"]
    return [case["v"] * d] + [s for _ in range(case["layers"]) for s in (d, 4 * d * d, d * d, d, 4 * d * d, 4 * d * d)] + [d]


def prepare(case, seed):
    g = _generator(seed)
    dt = DTYPES[case["dtype"]]
    op = case["op"]
    s = {"op": op, "dtype": dt}
    if op in ("loss", "grad"):
        n, v, d = case["n"], case["v"], case["d"]
        s["x"] = torch.randn(n, d, generator=g, device=DEV).to(dt)
        s["w"] = torch.empty(v, d, dtype=dt, device=DEV)
        for a in range(0, v, 16384):  # in pieces: the single-precision draws stay small
            b = min(v, a + 16384)
            s["w"][a:b] = (torch.randn(b - a, d, generator=g, device=DEV) * (2.0 / math.sqrt(d))).to(dt)
        s["labels"] = _without(_skewed(n, v, g), case["ignored"], g)
        s["weights"] = torch.rand(n, generator=g, device=DEV) + 0.5
        s["scale"] = (1024.0 if case["dtype"] == "fp16" else 1.0) / n  # half precision is trained with a scaled loss
    elif op == "embedding":
        n, v, d = case["n"], case["v"], case["d"]
        s["table"] = torch.randn(v, d, generator=g, device=DEV, dtype=dt)
        s["ids"] = _without(_skewed(n, v, g), case["ignored"], g)
        s["scale"] = math.sqrt(d)
    elif op == "embedding_grad":
        n, v, d = case["n"], case["v"], case["d"]
        s["rows"] = v
        s["grad"] = torch.randn(n, d, generator=g, device=DEV, dtype=dt)
        s["ids"] = _without(_skewed(n, v, g), case["ignored"], g)
        s["scale"] = 1.0 if case["dtype"] == "fp16" else math.sqrt(d)
    else:
        sizes = _clip_sizes(case)
        # tensors of one flat buffer, as programs keep them that exchange gradients; the optimiser's copy alike
        s["grads"] = torch.split(torch.randn(sum(sizes), generator=g, device=DEV, dtype=dt).mul_(0.01), sizes)
        s["flat"] = torch.empty(sum(sizes), dtype=dt, device=DEV)
        s["clipped"] = torch.split(s["flat"], sizes)
        s["max_norm"] = case["factor"] * 0.01 * math.sqrt(sum(sizes))
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _plain_loss(s):
    x, w = s["x"].float(), s["w"].float()
    logits = x @ w.T
    top = logits.amax(1, keepdim=True)
    lse = (top + (logits - top).exp().sum(1, keepdim=True).log()).squeeze(1)
    has = s["labels"] >= 0
    at = s["labels"].clamp(min=0).long().unsqueeze(1)
    none = torch.zeros_like(lse)
    loss = torch.where(has, lse - logits.gather(1, at).squeeze(1), none)
    lse = torch.where(has, lse, none)  # nothing of a row without a label
    return x, w, logits, lse, has, at, loss


def _plain(s):
    op, dt = s["op"], s["dtype"]
    if op == "loss":
        _, _, _, lse, _, _, loss = _plain_loss(s)
        return {"loss": loss, "lse": lse}
    if op == "grad":
        x, w, logits, lse, has, at, loss = _plain_loss(s)
        p = (logits - lse.unsqueeze(1)).exp_()
        p.scatter_add_(1, at, torch.full_like(lse, -1.0).unsqueeze(1))
        p *= torch.where(has, s["weights"] * s["scale"], torch.zeros_like(lse)).unsqueeze(1)
        return {"loss": loss, "lse": lse, "dx": (p @ w).to(dt), "dw": (p.T @ x).to(dt)}
    if op == "embedding":
        has = (s["ids"] >= 0).unsqueeze(1)
        out = s["table"][s["ids"].clamp(min=0)].float() * s["scale"]
        return {"out": torch.where(has, out, torch.zeros_like(out)).to(dt)}
    if op == "embedding_grad":
        has = (s["ids"] >= 0).unsqueeze(1)
        terms = torch.where(has, s["grad"].float(), torch.zeros((), device=DEV))
        total = torch.zeros(s["rows"], terms.shape[1], device=DEV).index_add_(0, s["ids"].clamp(min=0), terms)
        return {"dtable": (total * s["scale"]).to(dt)}
    flat = torch.cat(s["grads"]).float()
    norm = flat.square().sum(dtype=torch.float64).sqrt()
    flat *= torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0).float()
    return {"norm": norm.float(), "clipped": flat.to(dt)}


def _own(s):
    from paper_1909_04885_b200 import binding
    op = s["op"]
    if op == "loss":
        loss, lse = binding.softmax_loss(s["x"], s["w"], s["labels"])
        return {"loss": loss, "lse": lse}
    if op == "grad":
        loss, lse, dx, dw = binding.softmax_loss_grad(s["x"], s["w"], s["labels"], weights=s["weights"], scale=s["scale"])
        return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}
    if op == "embedding":
        return {"out": binding.embedding(s["table"], s["ids"], scale=s["scale"])}
    if op == "embedding_grad":
        return {"dtable": binding.embedding_grad(s["ids"], s["grad"], s["rows"], scale=s["scale"])}
    norm = binding.clip_gradients(s["grads"], s["max_norm"], out=s["clipped"])
    return {"norm": norm, "clipped": s["flat"]}


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op in ("loss", "grad"):
        n = case["n"]
        w = s["w"].double()
        loss, lse, dx = [], [], []
        dw = torch.zeros_like(w) if op == "grad" else None
        piece = max(1, min(n, (1 << 28) // case["v"]))
        for a in range(0, n, piece):
            x = s["x"][a:a + piece].double()
            y = s["labels"][a:a + piece].long()
            z = torch.mm(x, w.t())
            total = torch.logsumexp(z, dim=1)
            rows = torch.nonzero(y >= 0).flatten()
            of_label = torch.zeros_like(total)
            of_label[rows] = total[rows] - z[rows, y[rows]]
            lse.append(torch.where(y >= 0, total, torch.zeros_like(total)))
            loss.append(of_label)
            if op == "grad":
                c = torch.zeros_like(total)
                c[rows] = s["weights"][a:a + piece].double()[rows] * s["scale"]
                g = torch.softmax(z, dim=1)
                g[rows, y[rows]] -= 1.0
                g *= c[:, None]
                dx.append(torch.mm(g, w))
                dw.addmm_(g.t(), x)
        out = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
        if op == "grad":
            out |= {"dx": torch.cat(dx), "dw": dw}
        return out
    if op == "embedding":
        out = torch.zeros(case["n"], case["d"], dtype=torch.float64, device=DEV)
        rows = torch.nonzero(s["ids"] >= 0).flatten()
        out[rows] = s["table"][s["ids"][rows].long()].double() * s["scale"]
        return {"out": out}
    if op == "embedding_grad":
        rows = torch.nonzero(s["ids"] >= 0).flatten()
        out = torch.zeros(case["v"], case["d"], dtype=torch.float64, device=DEV)
        out.index_put_((s["ids"][rows].long(),), s["grad"][rows].double(), accumulate=True)
        return {"dtable": out * s["scale"]}
    square = sum(float(torch.dot(t.double(), t.double())) for t in s["grads"])
    norm = math.sqrt(square)
    c = min(1.0, s["max_norm"] / (norm + 1e-6))
    return {"norm": norm, "clipped": torch.cat([t.double() * c for t in s["grads"]])}


# ------------------------------------------------------------------------------------------------ work
def _distinct(n, v):
    """Expected distinct ids among n skewed ones."""
    r = np.arange(1, v + 1, dtype=np.float64)
    p = np.log1p(1.0 / r) / math.log(v + 1)
    return float(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def work(case):
    b = SIZE[case["dtype"]]
    op = case["op"]
    if op == "clip":
        k = sum(_clip_sizes(case))
        return {"bytes": 2.0 * b * k + 4, "flops": 3.0 * k}
    n, v, d = case["n"], case["v"], case["d"]
    if op == "loss":
        return {"bytes": b * (n + v) * d + 12.0 * n, "flops": 2.0 * n * v * d}
    if op == "grad":
        return {"bytes": 2.0 * b * (n + v) * d + 16.0 * n, "flops": 6.0 * n * v * d}
    if op == "embedding":
        return {"bytes": b * d * (_distinct(n, v) + n) + 4.0 * n, "flops": 1.0 * n * d}
    return {"bytes": b * d * (n + v) + 4.0 * n, "flops": 1.0 * n * d}
