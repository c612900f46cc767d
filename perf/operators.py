"""The 8-bit operators of a feed-forward block in training and serving, as a user calls them: what is measured, at which sizes.

norm        residual + root-mean-square norm, written in 8 bits with a scale per token;  norm_bwd  its backward pass
linear      product of 8-bit rows with scales per token and per channel;                 linear_bwd  its gradients, the
            input and the weight read in 8 bits
act         gated SiLU or GELU, written in 8 bits with a scale per token (serving);      act_train  the same with its
            input kept in 8 bits as a checkpoint, and the backward pass from that checkpoint

What is held in 8 bits comes back as the bf16 values that it stands for.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128          # columns per scale of a checkpoint
TINY = 2.0 ** -100   # rows and blocks below this are stored as zeros
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one token through the norm of a 1600-wide decoder: latency
        {"name": "norm one token", "kind": "norm", "t": 1, "d": 1600, "dtype": "bf16", "res": True},
        # a training batch of a 4096-wide model
        {"name": "norm batch", "kind": "norm", "t": 8192, "d": 4096, "dtype": "bf16", "res": True},
        # fp32 activations, odd width, no gradient that joins from the residual stream
        {"name": "norm backward odd fp32", "kind": "norm_bwd", "t": 1021, "d": 1277, "dtype": "fp32", "res": False},
        # 8 sequences of 1024 tokens of a 1600-wide decoder
        {"name": "norm backward batch", "kind": "norm_bwd", "t": 8192, "d": 1600, "dtype": "bf16", "res": True},
        # one token through the first product of the 1600-wide feed-forward: streams the weight
        {"name": "linear one token", "kind": "linear", "t": 1, "k": 1600, "n": 6400, "dtype": "bf16", "bias": False},
        # the 197 tokens of one image through a 768-wide encoder's projection, fp32 out
        {"name": "linear one image", "kind": "linear", "t": 197, "k": 768, "n": 2304, "dtype": "fp32", "bias": True},
        # a training batch
        {"name": "linear batch", "kind": "linear", "t": 8192, "k": 4096, "n": 8192, "dtype": "bf16", "bias": False},
        # ragged in every direction; fp32 gradients for fp32 master weights
        {"name": "linear backward odd", "kind": "linear_bwd", "t": 1003, "k": 769, "n": 1283, "dtype": "fp32", "bias": True},
        # 8 sequences of 1024 tokens through the first product of the 1600-wide feed-forward
        {"name": "linear backward batch", "kind": "linear_bwd", "t": 8192, "k": 1600, "n": 6400, "dtype": "bf16", "bias": False},
        # one token, serving
        {"name": "act one token", "kind": "act", "t": 1, "f": 6400, "dtype": "bf16", "gated": True},
        # a training batch of a gated feed-forward
        {"name": "act train batch", "kind": "act_train", "t": 8192, "f": 6400, "dtype": "bf16", "gated": True},
        # fp32 activations, odd width, not gated
        {"name": "act train odd fp32", "kind": "act_train", "t": 1003, "f": 5121, "dtype": "fp32", "gated": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width over its logarithm: of three, one a multiple of 64, one of 8 and one as it falls."""
    w, m = _log(rng, lo, hi), rng.choice((1, 8, 64))
    return max(m, w // m * m)


def draw(rng):
    kind = rng.choice(("norm", "norm_bwd", "linear", "linear_bwd", "act", "act_train"))
    c = {"kind": kind, "dtype": rng.choice(("bf16", "bf16", "fp32"))}
    if kind in ("norm", "norm_bwd"):
        c["d"] = _width(rng, 64, 8192)
        c["t"] = min(_log(rng, 1, 16384), 8192 * 4096 // c["d"])
        c["res"] = rng.random() < 0.75
    elif kind in ("linear", "linear_bwd"):
        c["k"], c["n"] = _width(rng, 64, 8192), _width(rng, 64, 16384)
        most = 8192 * (4096 * 8192 if kind == "linear" else 1600 * 6400)
        c["t"] = max(1, min(_log(rng, 1, 16384), most // (c["k"] * c["n"])))
        c["bias"] = rng.random() < 0.5
    else:
        c["f"] = _width(rng, 64, 16384)
        c["t"] = min(_log(rng, 1, 16384), 8192 * 6400 // c["f"])
        c["gated"] = rng.random() < 0.6
        if kind == "act_train" and c["dtype"] == "fp32":
            c["t"] = max(1, c["t"] // 2)
    return c


# ---- inputs --------------------------------------------------------------------------------------------------
def _rows8(x):
    """8-bit rows of x [rows, cols]: codes (row pitch a multiple of 16 bytes) and one scale per row."""
    rows, cols = x.shape
    amax = x.abs().amax(dim=1)
    zero = amax < TINY
    inv = torch.where(zero, 0.0, 127.0 / amax)
    pitch = (cols + 15) // 16 * 16
    q = torch.zeros(rows, pitch, dtype=torch.int8, device=x.device)
    q[:, :cols] = torch.round(x * inv[:, None]).to(torch.int8)
    return q[:, :cols], torch.where(zero, 0.0, amax / 127.0)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, device=dev, generator=gen)

    def hidden(t, d):
        """Hidden states: channels of different size, and a padding token of zeros in a batch."""
        x = normal(t, d) * torch.exp(0.5 * normal(d))
        if t > 16:
            x[t // 3] = 0.0
        return x

    s = {"case": case}
    kind, t = case["kind"], case["t"]
    if kind == "norm":
        d = case["d"]
        s["x"] = hidden(t, d).to(dt)
        s["res"] = (2.0 * hidden(t, d)).to(dt) if case["res"] else None
        s["weight"] = 1.0 + 0.1 * normal(d)
    elif kind == "norm_bwd":
        d = case["d"]
        s["h"] = (2.0 * hidden(t, d)).to(dt)
        s["rstd"] = torch.rsqrt(s["h"].float().square().mean(dim=1) + EPS)
        s["dy"] = (1e-3 * normal(t, d)).to(dt)
        s["dres"] = (1e-3 * normal(t, d)).to(dt) if case["res"] else None
        s["weight"] = 1.0 + 0.1 * normal(d)
    elif kind in ("linear", "linear_bwd"):
        k, n = case["k"], case["n"]
        s["x"], s["sx"] = _rows8(hidden(t, k))
        s["w"], s["sw"] = _rows8(0.02 * normal(n, k))
        if kind == "linear":
            s["bias"] = 0.02 * normal(n) if case["bias"] else None
        else:
            s["dy"] = (1e-3 * normal(t, n)).to(torch.bfloat16)
    else:
        f, parts = case["f"], 2 if case["gated"] else 1
        s["z"] = torch.cat([hidden(t, f) for _ in range(parts)], dim=1).to(dt)
        s["da"] = (1e-3 * normal(t, f)).to(dt) if kind == "act_train" else None
    return s


# ---- the plain forms: 32 bits, rounded once at the end ---------------------------------------------------------
def _values(y):
    """The values that the 8-bit rows of y stand for, and the scales."""
    amax = y.abs().amax(dim=-1, keepdim=True)
    zero = amax < TINY
    scale = torch.where(zero, torch.zeros_like(amax), amax / 127.0)
    q = torch.round(y * torch.where(zero, torch.zeros_like(amax), 127.0 / amax))
    return q * scale, scale


def _checkpoint(z):
    """z [t, f] through 8 bits and back, a scale per BLOCK columns."""
    t, f = z.shape
    full = torch.nn.functional.pad(z, (0, -f % BLOCK)).reshape(t, -1, BLOCK)
    return _values(full)[0].reshape(t, -1)[:, :f]


ROOT = math.sqrt(2.0 / math.pi)


def _act(g, u):
    if u is not None:
        return g / (1.0 + torch.exp(-g)) * u
    return 0.5 * g * (1.0 + torch.tanh(ROOT * (g + 0.044715 * g * g * g)))


def _act_grad(g, u, da):
    if u is not None:
        sig = 1.0 / (1.0 + torch.exp(-g))
        return torch.cat([da * u * sig * (1.0 + g * (1.0 - sig)), da * g * sig], dim=1)
    th = torch.tanh(ROOT * (g + 0.044715 * g * g * g))
    return da * (0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * ROOT * (1.0 + 3 * 0.044715 * g * g))


def _plain(s):
    case = s["case"]
    kind, dt = case["kind"], DT[case["dtype"]]
    if kind == "norm":
        h = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
        rstd = torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS)
        values, scale = _values(h * rstd * s["weight"])
        return [h.to(dt), values.to(torch.bfloat16), scale[:, 0], rstd[:, 0]]
    if kind == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh, wdy = s["h"].float() * rstd, s["weight"] * dy
        dx = rstd * (wdy - xh * (wdy * xh).mean(dim=1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return [dx.to(dt), (dy * xh).sum(dim=0)]
    if kind == "linear":
        out = (s["x"].float() @ s["w"].float().t()) * s["sx"][:, None] * s["sw"]
        return (out if s["bias"] is None else out + s["bias"]).to(dt)
    if kind == "linear_bwd":
        dy = s["dy"].float()
        out = [(dy @ (s["w"].float() * s["sw"][:, None])).to(dt), (dy.t() @ (s["x"].float() * s["sx"][:, None])).to(dt)]
        return out + [dy.sum(dim=0)] if case["bias"] else out
    z, f = s["z"].float(), case["f"]
    g, u = (z[:, :f], z[:, f:]) if case["gated"] else (z, None)
    values, scale = _values(_act(g, u))
    out = [values.to(torch.bfloat16), scale[:, 0]]
    if kind == "act_train":
        out.append(_act_grad(_checkpoint(g), None if u is None else _checkpoint(u), s["da"].float()).to(dt))
    return out


# ---- the framework's operators ---------------------------------------------------------------------------------
_kept = {}


def _own(s):
    if not _kept:
        from paper_2604_06836_b200 import q8, stq
        _kept.update(q8=q8, handle=stq.Handle())
    q8, handle = _kept["q8"], _kept["handle"]
    case = s["case"]
    kind, dt = case["kind"], DT[case["dtype"]]
    if kind == "norm":
        r = q8.norm(handle, s["x"], s["weight"], residual=s["res"], eps=EPS, values=True)
        return [r.h, r.values, r.rows.scale, r.rstd]
    if kind == "norm_bwd":
        return list(q8.norm_backward(handle, s["dy"], s["h"], s["weight"], s["rstd"], dres=s["dres"]))
    if kind in ("linear", "linear_bwd"):
        x, w = q8.Rows8(s["x"], s["sx"]), q8.Rows8(s["w"], s["sw"])
        if kind == "linear":
            return q8.linear(handle, x, w, bias=s["bias"], dtype=dt)
        out = [q8.linear_dx(handle, s["dy"], w, dtype=dt), q8.linear_dw(handle, s["dy"], x, dtype=dt)]
        return out + [q8.bias_grad(handle, s["dy"])] if case["bias"] else out
    act = "silu_gated" if case["gated"] else "gelu"
    r = q8.act(handle, s["z"], act, values=True, checkpoint=kind == "act_train")
    out = [r.values, r.rows.scale]
    if kind == "act_train":
        out.append(q8.act_backward(handle, s["da"], r.checkpoint))
    return out


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind, t = case["kind"], case["t"]
    e = 4 if case["dtype"] == "fp32" else 2
    if kind == "norm":        # x (and r) read, h, values and codes written
        d = case["d"]
        return {"bytes": t * d * (e * (3 if case["res"] else 1) + 3) + 4 * d + 8 * t, "flops": 8 * t * d}
    if kind == "norm_bwd":
        d = case["d"]
        return {"bytes": t * d * e * (4 if case["res"] else 3) + 8 * d + 4 * t, "flops": 12 * t * d}
    if kind == "linear":
        k, n = case["k"], case["n"]
        return {"bytes": t * k + n * k + t * n * e + 4 * (t + n), "flops": 2 * t * k * n}
    if kind == "linear_bwd":  # dy once for each product
        k, n = case["k"], case["n"]
        return {"bytes": 2 * t * n + (t + n) * k + (t + n) * k * e + 4 * (t + n), "flops": 4 * t * k * n}
    f, parts = case["f"], 2 if case["gated"] else 1
    read, written = t * f * parts * e, t * f * 3 + 4 * t
    if kind == "act_train":   # the checkpoint is written and read; da read, dz written
        saved = t * parts * (f + 4 * -(-f // BLOCK))
        return {"bytes": read + written + 2 * saved + t * f * e * (1 + parts), "flops": 40 * t * f}
    return {"bytes": read + written, "flops": 16 * t * f}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------
def _through8(y, width):
    """Every `width` columns of y [t, c] through 8 bits and back; and the scales [t, blocks]."""
    out, scales = torch.empty_like(y), []
    for at in range(0, y.shape[1], width):
        part = y[:, at:at + width]
        top = part.abs().max(dim=1).values
        step = torch.where(top < TINY, torch.zeros_like(top), top / 127)
        out[:, at:at + width] = torch.round(part / torch.where(step == 0, torch.ones_like(step), step)[:, None]) * step[:, None]
        scales.append(step)
    return out, torch.stack(scales, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    v = {n: x.double() for n, x in s.items() if torch.is_tensor(x)}
    kind = case["kind"]
    if kind == "norm":
        h = v["x"] + v["res"] if "res" in v else v["x"]
        rstd = (h.pow(2).mean(1) + EPS).pow(-0.5)
        values, scale = _through8(h * rstd[:, None] * v["weight"], case["d"])
        return [h, values, scale[:, 0], rstd]
    if kind == "norm_bwd":   # through the Jacobian's two terms
        n = case["d"]
        up = v["dy"] * v["weight"]
        dot = (up * v["h"]).sum(1)
        dx = up * v["rstd"][:, None] - v["h"] * (v["rstd"].pow(3) * dot / n)[:, None]
        return [dx + v["dres"] if "dres" in v else dx, (v["dy"] * v["h"] * v["rstd"][:, None]).sum(0)]
    if kind == "linear":
        out = torch.matmul(v["x"] * v["sx"][:, None], (v["w"] * v["sw"][:, None]).T)
        return out + v["bias"] if "bias" in v else out
    if kind == "linear_bwd":
        out = [torch.matmul(v["dy"] * v["sw"], v["w"]), torch.matmul((v["dy"] * v["sx"][:, None]).T, v["x"])]
        return out + [v["dy"].sum(0)] if case["bias"] else out
    f = case["f"]
    z = v["z"]
    gelu = lambda x: x * torch.sigmoid(2 * ROOT * (x + 0.044715 * x ** 3))  # noqa: E731
    a = z[:, :f] * torch.sigmoid(z[:, :f]) * z[:, f:] if case["gated"] else gelu(z)
    values, scale = _through8(a, f)
    if kind == "act":
        return [values, scale[:, 0]]
    # the derivative at the checkpoint, by the product rule
    kept = torch.cat([_through8(part, BLOCK)[0] for part in z.split(f, dim=1)], dim=1)
    g = kept[:, :f]
    if case["gated"]:
        sig = torch.sigmoid(g)
        dz = torch.cat([v["da"] * kept[:, f:] * (sig + g * sig * torch.sigmoid(-g)), v["da"] * g * sig], dim=1)
    else:
        inner = 2 * ROOT * (g + 0.044715 * g ** 3)
        sig = torch.sigmoid(inner)
        dz = v["da"] * (sig + g * sig * torch.sigmoid(-inner) * 2 * ROOT * (1 + 3 * 0.044715 * g ** 2))
    return [values, scale[:, 0], dz]
