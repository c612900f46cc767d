"""The operators at the end of a training step, as a user calls them: what is measured, at which sizes.

score       cross entropy of tokens over a vocabulary, from the last hidden states and the output matrix, without gradients
train       the same and its gradients: of the hidden states, of the matrix and of its bias
norm        the 2-norm of all gradients together, with the factor that clips them
clip        the same, and the clipped gradients

The logits of a whole batch (up to 8192 x 50257 here) exist in the plain forms only.
"""
import math

import torch

own = False

IGNORE = -100
EPS = 1e-6
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # the score of one token of a 1600-wide decoder: streams the matrix
        {"name": "score one token", "kind": "score", "t": 1, "d": 1600, "v": 50257, "bias": False, "masked": 0.0},
        # candidates that a ranker compares; nothing is a whole number of tiles
        {"name": "score odd", "kind": "score", "t": 61, "d": 769, "v": 1283, "bias": True, "masked": 0.1},
        # evaluation of 8 sequences of 1024 tokens
        {"name": "score batch", "kind": "score", "t": 8192, "d": 1600, "v": 50257, "bias": False, "masked": 0.0},
        # a batch of images over 1000 classes
        {"name": "train classes", "kind": "train", "t": 512, "d": 768, "v": 1000, "bias": True, "masked": 0.0, "dw": "fp32"},
        # ragged in every direction, padding in the batch
        {"name": "train odd", "kind": "train", "t": 1003, "d": 1025, "v": 5121, "bias": False, "masked": 0.2, "dw": "bf16"},
        # masked language model: 85 % of 8 x 512 tokens have no loss; fp32 gradients for fp32 master weights
        {"name": "train masked", "kind": "train", "t": 4096, "d": 1024, "v": 50265, "bias": True, "masked": 0.85, "dw": "fp32"},
        # 8 sequences of 1024 tokens
        {"name": "train batch", "kind": "train", "t": 8192, "d": 1600, "v": 50257, "bias": False, "masked": 0.0, "dw": "bf16"},
        # a small model's tensors: latency
        {"name": "norm small", "kind": "norm", "layers": 2, "d": 136, "v": 777, "dtype": "fp32", "scale": 1.0},
        # all tensors of a decoder of 1.5 billion parameters
        {"name": "norm large", "kind": "norm", "layers": 48, "d": 1600, "v": 50257, "dtype": "bf16", "scale": 1.0},
        # odd lengths throughout, bf16 gradients kept as they are
        {"name": "clip odd", "kind": "clip", "layers": 3, "d": 237, "v": 1283, "dtype": "bf16", "out": "bf16", "scale": 1.0},
        # fp16 gradients under a loss scale to the fp32 gradients of the master weights, 355 million
        {"name": "clip scaled", "kind": "clip", "layers": 24, "d": 1024, "v": 50257, "dtype": "fp16", "out": "fp32", "scale": 4096.0},
        # fp32 gradients of 774 million parameters
        {"name": "clip large", "kind": "clip", "layers": 36, "d": 1280, "v": 50257, "dtype": "fp32", "out": "fp32", "scale": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over its logarithm: of three, one a multiple of 64, one of 8 and one as it falls."""
    w, m = _log(rng, lo, hi), rng.choice((1, 8, 64))
    return max(m, w // m * m)


def draw(rng):
    kind = rng.choice(("score", "score", "train", "train", "norm", "clip"))
    c = {"kind": kind}
    if kind in ("score", "train"):
        c["d"], c["v"] = _width(rng, 64, 4096), _width(rng, 100, 131072)
        c["t"] = max(1, min(_log(rng, 1, 16384), 8192 * 1600 * 50257 // (c["d"] * c["v"])))
        c["bias"] = rng.random() < 0.4
        c["masked"] = rng.choice((0.0, 0.1, 0.85))
        if kind == "train":
            c["dw"] = rng.choice(("bf16", "bf16", "fp32"))
            if c["dw"] == "fp32":
                c["t"] = max(1, c["t"] // 2)
    else:
        c["d"] = _width(rng, 32, 1600)
        most = 1_500_000_000 if kind == "norm" else 600_000_000
        c["layers"] = max(1, min(_log(rng, 1, 48), most // (12 * c["d"] * c["d"])))
        c["v"] = _width(rng, 100, 50257)
        c["dtype"] = rng.choice(("bf16", "fp16", "fp32"))
        if kind == "clip":
            c["out"] = rng.choice((c["dtype"], "fp32"))
        c["scale"] = 4096.0 if c["dtype"] == "fp16" else 1.0
    return c


# ---- inputs --------------------------------------------------------------------------------------------------
def _lengths(case):
    """Lengths of a decoder's tensors: embeddings, then per layer two norms and four products with their biases."""
    d = case["d"]
    layer = [d, d, 3 * d * d, 3 * d, d * d, d, d, d, 4 * d * d, 4 * d, 4 * d * d, d]
    return [case["v"] * d, 1024 * d] + case["layers"] * layer + [d, d]


def _many(case, seed, dev, gen):
    dt, n = DT[case["dtype"]], _lengths(case)
    grads, at = [], 0
    size = 10.0 ** (-5.0 + 3.0 * torch.rand(len(n), generator=torch.Generator().manual_seed(seed)))   # 1e-5 .. 1e-2
    for i, k in enumerate(n):
        g = torch.randn(k, device=dev, generator=gen)
        if i == 0:      # the embedding: tokens that the batch does not hold have no gradient
            g.view(case["v"], -1)[case["v"] // 4:] = 0.0
        grads.append(g.mul_(float(size[i]) * case["scale"]).to(dt))
    s = {"grads": grads, "inv": None if case["scale"] == 1.0 else torch.full((1,), 1.0 / case["scale"], device=dev)}
    if case["kind"] == "clip":      # the results lie in one buffer, each tensor on a boundary of 64 elements
        starts = []
        for k in n:
            starts.append(at)
            at += -(-k // 64) * 64
        s["flat"] = torch.zeros(at, device=dev, dtype=DT[case["out"]])
        s["out"] = [s["flat"][a:a + k] for a, k in zip(starts, n)]
    return s


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    if case["kind"] in ("norm", "clip"):
        return {"case": case, "max_norm": 1.0, **_many(case, seed, dev, gen)}
    t, d, v = case["t"], case["d"], case["v"]

    def uniform(n):
        return torch.rand(n, device=dev, generator=gen)

    w = (0.02 * torch.randn(v, d, device=dev, generator=gen)).to(torch.bfloat16)
    target = (v * uniform(t) ** 3).long().clamp_(max=v - 1)      # a few tokens are frequent
    # hidden states that a trained model has: the logit of the target is up to 8 above what it were otherwise
    x = torch.randn(t, d, device=dev, generator=gen) + (8.0 / (0.0004 * d)) * uniform(t)[:, None] * w[target].float()
    if case["masked"]:
        target[uniform(t) < case["masked"]] = IGNORE
        target[t // 2] = IGNORE if t > 1 else target[0]
    s = {"case": case, "x": x.to(torch.bfloat16), "w": w, "target": target}
    s["bias"] = 0.1 * torch.randn(v, device=dev, generator=gen) if case["bias"] else None
    if case["kind"] == "train":      # the gradient of the mean over the tokens that count
        s["dloss"] = torch.full((t,), 1.0 / max(1, int((target != IGNORE).sum())), device=dev)
    return s


# ---- the plain forms: 32 bits (the norm's sum 64), rounded once at the end ---------------------------------------
def _plain_loss(s):
    case, target = s["case"], s["target"]
    x, w = s["x"].float(), s["w"].float()
    logits = x @ w.t()
    if s["bias"] is not None:
        logits += s["bias"]
    top = logits.max(dim=1, keepdim=True).values
    lse = top + torch.log(torch.exp(logits - top).sum(dim=1, keepdim=True))
    counts = target != IGNORE      # (the others have neither a loss nor a normaliser)
    row, column = torch.arange(case["t"], device=x.device), torch.where(counts, target, 0)
    loss = torch.where(counts, lse[:, 0] - logits[row, column], 0.0)
    out = [loss, torch.where(counts, lse[:, 0], 0.0)]
    if case["kind"] == "score":
        return out
    p = torch.exp(logits - lse)
    p[row, column] -= 1.0
    p *= torch.where(counts, s["dloss"], 0.0)[:, None]
    out += [(p @ w).to(torch.bfloat16), (p.t() @ x).to(DT[case["dw"]])]
    return out + [p.sum(dim=0)] if case["bias"] else out


def _plain_norm(s):
    flat = torch.cat(s["grads"]).float()
    norm = flat.square().sum(dtype=torch.float64).sqrt().float()
    if s["inv"] is not None:
        norm = norm * s["inv"][0]
    factor = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    if s["inv"] is not None:
        factor = factor * s["inv"][0]
    if s["case"]["kind"] == "norm":
        return [norm, factor]
    torch._foreach_copy_(s["out"], list((flat * factor).to(s["flat"].dtype).split(_lengths(s["case"]))))
    return [norm, s["flat"]]


# ---- the framework's operators -----------------------------------------------------------------------------------
_kept = {}


def _own(s):
    if not _kept:
        from paper_2604_06836_b200 import clip, stq, vocab
        _kept.update(clip=clip, vocab=vocab, handle=stq.Handle())
    clip, vocab, handle = _kept["clip"], _kept["vocab"], _kept["handle"]
    kind = s["case"]["kind"]
    if kind == "norm":
        r = clip.grad_norm(handle, s["grads"], max_norm=s["max_norm"], inv_scale=s["inv"])
        return [r.norm, r.factor]
    if kind == "clip":
        r = clip.clip_grads(handle, s["grads"], s["max_norm"], inv_scale=s["inv"], out=s["out"])
        return [r.norm, s["flat"]]
    r = vocab.loss(handle, s["x"], s["w"], s["target"], bias=s["bias"], ignore_index=IGNORE)
    if kind == "score":
        return [r.loss, r.lse]
    g = vocab.loss_backward(handle, s["dloss"], s["x"], s["w"], s["target"], r.lse, bias=s["bias"], ignore_index=IGNORE,
                            dtype=DT[s["case"]["dw"]])
    return [r.loss, r.lse, g.dx, g.dw] + ([g.dbias] if s["case"]["bias"] else [])


def run(state):
    if own:
        return _own(state)
    return _plain_norm(state) if state["case"]["kind"] in ("norm", "clip") else _plain_loss(state)


def work(case):
    e = {n: 4 if n == "fp32" else 2 for n in DT}
    if case["kind"] in ("norm", "clip"):
        n = sum(_lengths(case))
        written = e[case["out"]] if case["kind"] == "clip" else 0
        return {"bytes": n * (e[case["dtype"]] + written), "flops": (3 if written else 2) * n}
    t, d, v = case["t"], case["d"], case["v"]
    real = max(1, round(t * (1.0 - case["masked"])))      # tokens that count: nothing is computed of the others
    read = 2 * (real + v) * d + 8 * t + (4 * v if case["bias"] else 0)
    if case["kind"] == "score":
        return {"bytes": read + 8 * t, "flops": 2 * real * v * d}
    written = 8 * t + 2 * t * d + e[case["dw"]] * v * d + (4 * v if case["bias"] else 0)
    return {"bytes": read + 4 * real + written, "flops": 6 * real * v * d}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "clip"):
        inv = 1.0 / case["scale"]
        norm = math.sqrt(sum(float(torch.dot(part, part)) for g in s["grads"] for part in g.double().split(1 << 28))) * inv
        factor = min(1.0, 1.0 / (norm + EPS)) * inv
        if case["kind"] == "norm":
            return [torch.tensor(norm, dtype=torch.float64), torch.tensor(factor, dtype=torch.float64)]
        flat = torch.zeros(s["flat"].numel(), device="cuda", dtype=torch.float64)
        for g, o in zip(s["grads"], s["out"]):
            flat[o.storage_offset():o.storage_offset() + o.numel()] = g.double() * factor
        return [torch.tensor(norm, dtype=torch.float64), flat]
    x, w = s["x"].double(), s["w"].double()
    loss, lse, dx = [], [], []
    dw, db = torch.zeros_like(w), torch.zeros_like(w[:, 0])
    for at in range(0, case["t"], 2048):      # tokens by the block, differentiated through the definition's Jacobian
        xs, target = x[at:at + 2048], s["target"][at:at + 2048]
        z = torch.einsum("td,vd->tv", xs, w)
        if case["bias"]:
            z = z + s["bias"].double()
        total = torch.logsumexp(z, dim=1)
        real = (target >= 0).double()
        loss.append((total - z.gather(1, target.clamp(min=0)[:, None])[:, 0]) * real)
        lse.append(total * real)
        if case["kind"] == "train":
            dz = torch.softmax(z, dim=1)
            dz.scatter_add_(1, target.clamp(min=0)[:, None], -torch.ones(len(xs), 1, dtype=dz.dtype, device=dz.device))
            dz *= (real * s["dloss"][at:at + 2048].double())[:, None]
            dx.append(torch.mm(dz, w))
            dw.addmm_(dz.T, xs)
            db += dz.sum(0)
    out = [torch.cat(loss), torch.cat(lse)]
    if case["kind"] == "train":
        out += [torch.cat(dx), dw] + ([db] if case["bias"] else [])
    return out
