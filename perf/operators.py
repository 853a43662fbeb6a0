"""The operators of a transformer's feed-forward block as measured cases: layer norm, the linear layer with bias, activation and
residual, and the linear layer of rows sorted by expert, each forward and with its gradients.

`own` false: the plain form, elementary torch operations in 32 bits, rounded once at the end.  `own` true: this package's calls.
A training pass runs the forward operator and then the backward one, whose z is an input of its own, as a schedule that
alternates micro-batches has them: the forward's, and the one that the micro-batch whose turn it is stored.
Formulas (x rows of `cin` features, W [cout][cin], z stored in the operands' type for the backward pass):

    linear    z = x W^T + b,  y = act(z) + r;     dz = dy act'(z),  dx = dz W,  dW = dz^T x,  db = sum of dz over rows
    experts   the same, rows offsets[g] .. offsets[g+1] - 1 with W[g] and b[g]
    norm      m = mean(x), s = (mean((x - m)^2) + eps)^-1/2, h = (x - m) s, y = h gamma + beta;
              with g = dy gamma: dx = s (g - mean(g) - h mean(g h)),  dgamma = sum of dy h,  dbeta = sum of dy
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-5
LARGEST = 6 * 8192 * 2048 * 8192        # operations of the largest listed case


def _norm(rows, features, dtype, train):
    return dict(op="norm", rows=rows, features=features, dtype=dtype, train=train)


def _linear(rows, cin, cout, dtype, act, bias, residual, train, groups=0):
    return dict(op="experts" if groups else "linear", rows=rows, cin=cin, cout=cout, groups=groups, dtype=dtype, act=act, bias=bias, residual=residual,
                train=train)


def listed():
    return [
        # one token while answering: the latency of a call
        dict(_norm(1, 4096, "bf16", False), name="norm_token"),
        # a long prompt, or several packed ones
        dict(_norm(16384, 4096, "bf16", False), name="norm_prompt"),
        # a training step's tokens in a wide model
        dict(_norm(8192, 8192, "bf16", True), name="norm_train"),
        # a small model in full precision, no size a power of two
        dict(_norm(1537, 1000, "f32", True), name="norm_train_odd_f32"),
        # one token through an up projection
        dict(_linear(1, 4096, 4096, "bf16", "gelu", True, False, False), name="linear_token"),
        # a prompt through a layer whose output joins the residual stream
        dict(_linear(4096, 4096, 4096, "bf16", "gelu_tanh", True, True, False), name="linear_prompt"),
        # a training step of the up projection
        dict(_linear(8192, 2048, 8192, "bf16", "silu", True, False, True), name="linear_train"),
        # a small layer in full precision with sizes that fit no tile and no vector
        dict(_linear(1000, 777, 1283, "f32", "relu", True, True, True), name="linear_train_odd_f32"),
        # a few tokens, each with two of many experts
        dict(_linear(16, 2048, 1024, "bf16", "silu", False, False, False, 64), name="experts_token"),
        # a prompt's tokens sorted by expert, unevenly spread
        dict(_linear(8192, 2048, 4096, "bf16", "silu", False, False, False, 32), name="experts_prompt"),
        # a training step of a layer of experts
        dict(_linear(4096, 1024, 2048, "bf16", "gelu", True, False, True, 16), name="experts_train"),
        # a small layer of experts in full precision, odd rows
        dict(_linear(777, 200, 328, "f32", "relu", True, False, True, 5), name="experts_train_odd_f32"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """A feature count: mostly whole vectors, as models have them, sometimes any number."""
    n = _log(rng, low, high)
    return n if rng.random() < 0.25 else max(8, n // 8 * 8)


def draw(rng):
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    train = rng.random() < 0.5
    if rng.random() < 0.3:
        while True:
            rows, features = _log(rng, 1, 32768), _width(rng, 16, 16384)
            if rows * features <= 64 << 20:
                return _norm(rows, features, dtype, train)
    groups = rng.choice([0, rng.randint(2, 64)])
    while True:
        rows, cin, cout = _log(rng, 1, 16384), _width(rng, 32, 8192), _width(rng, 32, 8192)
        # full precision costs the plain form as much, and gradients are two more products; all experts' weights are there, used or not
        if rows * cin * cout * (6 if train else 2) <= (LARGEST if dtype == "bf16" else LARGEST // 8) and max(1, groups) * cin * cout <= 128 << 20:
            return _linear(rows, cin, cout, dtype, rng.choice(ACTIVATIONS), rng.random() < 0.6, rng.random() < 0.4, train, groups)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, device="cuda", dtype=dtype)

    s = dict(case=case)
    rows = case["rows"]
    if case["op"] == "norm":
        c = case["features"]
        s["x"] = normal(rows, c, scale=1.5)
        s["x"] += 0.25
        s["gamma"], s["beta"] = 1 + normal(c, scale=0.2, dtype=torch.float32), normal(c, scale=0.2, dtype=torch.float32)
        s["y"], s["mean"], s["rstd"] = empty(rows, c), empty(rows, dtype=torch.float32), empty(rows, dtype=torch.float32)
        if case["train"]:
            s["dy"] = normal(rows, c)
            s["dx"], s["dgamma"], s["dbeta"] = empty(rows, c), empty(c, dtype=torch.float32), empty(c, dtype=torch.float32)
        if own:
            from paper_1903_06498_amd.binding import StripeNorm
            s["op"] = StripeNorm(rows, c, case["dtype"], eps=EPS)
    else:
        k, n, e = case["cin"], case["cout"], case["groups"]
        lead = (e,) if e else ()
        s["x"], s["w"] = normal(rows, k), normal(*lead, n, k, scale=k ** -0.5)
        s["bias"] = normal(*lead, n, scale=0.1, dtype=torch.float32) if case["bias"] else None
        s["residual"] = normal(rows, n) if case["residual"] else None
        s["offsets"] = None
        if e:
            # an uneven share for each expert, and none for some
            r = np.random.RandomState(seed % (1 << 32))
            share = r.gamma(2.0, size=e) * (r.rand(e) > 0.1) + 1e-9
            s["counts"] = r.multinomial(rows, share / share.sum())
            ends = torch.from_numpy(np.concatenate([[0], np.cumsum(s["counts"])]).astype(np.int32))
            s["offsets"] = ends.cuda()
        s["y"] = empty(rows, n)
        s["pre"] = empty(rows, n) if case["train"] and case["act"] != "none" else None
        if case["train"]:
            s["dy"] = normal(rows, n)
            s["z"] = normal(rows, n) if s["pre"] is not None else None
            s["dx"], s["dw"], s["dbias"] = empty(rows, k), empty(*lead, n, k), empty(*lead, n, dtype=torch.float32) if case["bias"] else None
        if own:
            from paper_1903_06498_amd.binding import StripeLinear
            s["op"] = StripeLinear(rows, k, n, case["dtype"], activation=case["act"], groups=e)
    if own and s["op"].workspace_bytes:
        s["op"].set_workspace(torch.empty(s["op"].workspace_bytes, dtype=torch.uint8, device="cuda"))
    return s


# ---- the package's calls ---------------------------------------------------
def _run_own(s):
    case, op = s["case"], s["op"]
    if case["op"] == "norm":
        op.run(s["x"], s["y"], gamma=s["gamma"], beta=s["beta"], mean=s["mean"], rstd=s["rstd"])
        out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        if case["train"]:
            op.backward(s["dy"], s["x"], s["mean"], s["rstd"], gamma=s["gamma"], dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
            out.update(dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
        return out
    op.run(s["x"], s["w"], s["y"], bias=s["bias"], residual=s["residual"], offsets=s["offsets"], pre=s["pre"])
    out = {"y": s["y"]}
    if s["pre"] is not None:
        out["pre"] = s["pre"]
    if case["train"]:
        op.backward(s["dy"], s["x"], s["w"], pre=s["z"], offsets=s["offsets"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"])
        out.update(dx=s["dx"], dw=s["dw"])
        if s["dbias"] is not None:
            out["dbias"] = s["dbias"]
    return out


# ---- the plain form --------------------------------------------------------
def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _slots(s):
    """Each row's place in a padded [groups][longest group] layout, and its group."""
    group = torch.searchsorted(s["offsets"][1:], torch.arange(s["case"]["rows"], device="cuda", dtype=torch.int32), right=True)
    longest = int(s["counts"].max())
    return group, group * longest + torch.arange(s["case"]["rows"], device="cuda") - s["offsets"][group], longest


def _padded(rows, at, groups, longest):
    out = torch.zeros(groups * longest, rows.shape[1], device="cuda")
    out[at] = rows
    return out.view(groups, longest, rows.shape[1])


def _run_plain(s):
    case = s["case"]
    dt = TYPES[case["dtype"]]
    x = s["x"].float()
    if case["op"] == "norm":
        mean = x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt(((x - mean) * (x - mean)).mean(1, keepdim=True) + EPS)
        h = (x - mean) * rstd
        out = {"y": (h * s["gamma"] + s["beta"]).to(dt), "mean": mean[:, 0], "rstd": rstd[:, 0]}
        if case["train"]:
            dy = s["dy"].float()
            g = dy * s["gamma"]
            dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
            out.update(dx=dx.to(dt), dgamma=(dy * h).sum(0), dbeta=dy.sum(0))
        return out
    w, e = s["w"].float(), case["groups"]
    if e:
        group, at, longest = _slots(s)
        xp = _padded(x, at, e, longest)
        z = torch.bmm(xp, w.transpose(1, 2).contiguous()).view(e * longest, -1)[at]
        if s["bias"] is not None:
            z = z + s["bias"][group]
    else:
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"]
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(dt)}
    if s["pre"] is not None:
        out["pre"] = z.to(dt)
    if case["train"]:
        dz = s["dy"].float()
        if s["z"] is not None:
            dz = dz * _slope(s["z"].float(), case["act"])
        if e:
            dp = _padded(dz, at, e, longest)
            dx, dw = torch.bmm(dp, w).view(e * longest, -1)[at], torch.bmm(dp.transpose(1, 2).contiguous(), xp)
        else:
            dx, dw = dz @ w, dz.t() @ x
        out.update(dx=dx.to(dt), dw=dw.to(dt))
        if s["dbias"] is not None:
            out["dbias"] = dp.sum(1) if e else dz.sum(0)
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    size, m = SIZE[case["dtype"]], case["rows"]
    if case["op"] == "norm":
        c = case["features"]
        moved, flops = size * 2 * m * c + 8 * m + 8 * c, 8 * m * c
        if case["train"]:       # the forward's outputs and the statistics stay for a backward that reads x and dy
            moved, flops = moved + size * 3 * m * c + 8 * m + 12 * c, flops + 14 * m * c
        return {"bytes": moved, "flops": flops}
    k, n, e = case["cin"], case["cout"], case["groups"]
    used = min(max(1, e), m)      # weight matrices that some row meets, at most
    moved = size * (m * k + used * n * k + m * n * (2 if case["residual"] else 1)) + (4 * used * n if case["bias"] else 0)
    flops = 2 * m * n * k
    if case["train"]:
        with_pre = case["act"] != "none"
        moved += size * (m * n * (3 if with_pre else 1) + 2 * m * k + (used + max(1, e)) * n * k) + (4 * max(1, e) * n if case["bias"] else 0)
        flops *= 3
    return {"bytes": moved, "flops": flops}


# ---- the definition in 64 bits ---------------------------------------------
def _exact_act(z, name):
    """Value and derivative."""
    if name == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros_like(z))
    if name == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":      # 1/2 (1 + tanh(u)) = sigmoid(2u)
        u2 = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z.pow(3))
        p = torch.sigmoid(u2)
        return z * p, p + z * p * (1 - p) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z.square())
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    return z, torch.ones_like(z)


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"] == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS).rsqrt()
        h = (x - mean[:, None]) * rstd[:, None]
        out = {"y": torch.addcmul(s["beta"].double(), h, s["gamma"].double()), "mean": mean, "rstd": rstd}
        if case["train"]:
            dy = s["dy"].double()
            g, c = dy * s["gamma"].double(), case["features"]
            dot = (g * h).sum(1) / c
            out["dx"] = (g - (g.sum(1) / c)[:, None] - h * dot[:, None]) * rstd[:, None]
            out["dgamma"], out["dbeta"] = torch.einsum("rc,rc->c", dy, h), torch.einsum("rc->c", dy)
        return out
    ends = s["offsets"].tolist() if case["groups"] else [0, case["rows"]]
    w = s["w"].double() if case["groups"] else s["w"].double()[None]
    bias = None if s["bias"] is None else s["bias"].double().view(len(ends) - 1, -1)
    z = x.new_zeros(case["rows"], case["cout"])
    for g, (a, b) in enumerate(zip(ends, ends[1:])):
        z[a:b] = torch.mm(x[a:b], w[g].t())
        if bias is not None:
            z[a:b] += bias[g]
    out = {"y": _exact_act(z, case["act"])[0]}
    if s["residual"] is not None:
        out["y"] = out["y"] + s["residual"].double()
    if s["pre"] is not None:
        out["pre"] = z
    if case["train"]:
        dz = s["dy"].double()
        if s["z"] is not None:
            dz = dz * _exact_act(s["z"].double(), case["act"])[1]
        dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), x.new_zeros(len(ends) - 1, case["cout"])
        for g, (a, b) in enumerate(zip(ends, ends[1:])):
            dx[a:b], dw[g], db[g] = torch.mm(dz[a:b], w[g]), torch.mm(dz[a:b].t(), x[a:b]), dz[a:b].sum(0)
        out["dx"], out["dw"] = dx, dw.view(s["w"].shape)
        if s["bias"] is not None:
            out["dbias"] = db.view(s["bias"].shape)
    return out
