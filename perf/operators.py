"""Cases of the operators a training step runs around its quantized matrix products, with their plain forms:

  xent  linear + softmax cross entropy over a large vocabulary: loss, and the gradients of activations and weights
  gn    group norm with an activation on channels-last activations, forward and backward
  clip  the norm over all gradients of a model, and clipping by it

`run` computes the plain form (elementary torch operations in 32 bits, rounded once at the end) while `own` is
false, and calls the library while it is true.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}
IGNORE = -100
EPS = 1e-5        # of the group norm's variance
CLIP_EPS = 1e-6   # added to the norm before the division

# parameter sizes of the 32x32-image network (3x3 stem, four stages of two blocks, linear head): what its step clips
CNN_WIDTHS, CNN_CLASSES = (64, 128, 256, 512), 100


def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _generator(seed):
    g = torch.Generator(device=_device())
    g.manual_seed(seed)
    return g


# ---- cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # the head of the 100-class image network on one batch: a call that is all latency, weights stored [D, V]
        {"name": "xent_cnn_head", "op": "xent", "mode": "train", "tokens": 128, "features": 512, "classes": 100,
         "dtype": "fp32", "w_is_cd": False},
        # score of one token against a full vocabulary: reading the weights once is all there is
        {"name": "xent_one_token", "op": "xent", "mode": "loss", "tokens": 1, "features": 2048, "classes": 32000,
         "dtype": "bf16", "w_is_cd": True},
        # ragged batch, odd vocabulary, a weight for each token's loss that is known only when the gradient is asked for
        {"name": "xent_rows_odd", "op": "xent", "mode": "rows", "tokens": 1531, "features": 1000, "classes": 50257,
         "dtype": "bf16", "w_is_cd": True},
        # an ordinary training micro-batch
        {"name": "xent_mid", "op": "xent", "mode": "train", "tokens": 4096, "features": 2048, "classes": 32000,
         "dtype": "bf16", "w_is_cd": True},
        # the same loss for a model held in 32 bits throughout, weights stored [D, V]
        {"name": "xent_fp32", "op": "xent", "mode": "train", "tokens": 2048, "features": 1024, "classes": 32768,
         "dtype": "fp32", "w_is_cd": False},
        # the largest: a long batch and a large vocabulary
        {"name": "xent_large", "op": "xent", "mode": "train", "tokens": 8192, "features": 4096, "classes": 131072,
         "dtype": "bf16", "w_is_cd": True},
        # last and first stage of the image network at its batch of 128
        {"name": "gn_cnn_late", "op": "gn", "mode": "train", "batch": 128, "height": 4, "width": 4, "channels": 512,
         "groups": 32, "dtype": "fp32", "param": "fp32", "act": "relu"},
        {"name": "gn_cnn_early", "op": "gn", "mode": "train", "batch": 128, "height": 32, "width": 32, "channels": 64,
         "groups": 32, "dtype": "fp32", "param": "fp32", "act": "relu"},
        # inference on odd sizes in half precision
        {"name": "gn_infer_odd", "op": "gn", "mode": "infer", "batch": 7, "height": 57, "width": 43, "channels": 90,
         "groups": 9, "dtype": "fp16", "param": "fp32", "act": "relu"},
        # training on large feature maps
        {"name": "gn_large", "op": "gn", "mode": "train", "batch": 16, "height": 128, "width": 128, "channels": 512,
         "groups": 32, "dtype": "bf16", "param": "fp32", "act": "silu"},
        # the gradients of the image network's step
        {"name": "clip_cnn", "op": "clip", "model": "cnn", "count": 62, "total": 0, "dtype": "fp32", "norm": "2",
         "shapes": 0},
        # a larger model's gradients, some tensors in 16 bits and some in 32, sizes from one element to many millions
        {"name": "clip_large", "op": "clip", "model": "ragged", "count": 60, "total": 400_000_000, "dtype": "mixed",
         "norm": "2", "shapes": 7},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("xent", "xent", "gn", "gn", "clip"))
    if op == "xent":
        dtype = rng.choice(("bf16", "bf16", "fp32"))
        most = 1 << (42 if dtype == "bf16" else 36)
        while True:
            t, d, v = _log_int(rng, 1, 8192), _log_int(rng, 48, 4096), _log_int(rng, 12, 131072)
            if rng.random() < 0.5:       # most models keep multiples of 8; the rest is any number
                d, v = -(-d // 8) * 8, -(-v // 8) * 8
            if t * d * v <= most:
                break
        return {"op": op, "mode": rng.choice(("train", "train", "rows", "loss")), "tokens": t, "features": d,
                "classes": v, "dtype": dtype, "w_is_cd": rng.random() < 0.6}
    if op == "gn":
        dtype = rng.choice(("fp32", "bf16", "fp16"))
        while True:
            b, h, w = _log_int(rng, 1, 128), _log_int(rng, 1, 128), _log_int(rng, 1, 128)
            groups = rng.choice((1, 2, 4, 8, 9, 16, 32))
            c = groups * _log_int(rng, 1, max(1, 512 // groups))
            if 1 << 12 <= b * h * w * c <= 1 << 27 and h * w * c // groups >= 8:
                break
        return {"op": op, "mode": rng.choice(("train", "train", "infer")), "batch": b, "height": h, "width": w,
                "channels": c, "groups": groups, "dtype": dtype,
                "param": rng.choice(("fp32", "fp32", dtype)), "act": rng.choice(("none", "relu", "silu"))}
    return {"op": op, "model": "ragged", "count": rng.randint(1, 60), "total": _log_int(rng, 1000, 400_000_000),
            "dtype": rng.choice(("fp32", "bf16", "fp16", "mixed")), "norm": rng.choice(("2", "2", "2", "inf")),
            "shapes": rng.randrange(1 << 20)}


def _clip_shapes(case):
    """[(size, dtype name)] of the gradients, from the case alone."""
    if case["model"] == "cnn":
        sizes, cin = [CNN_WIDTHS[0] * 27, CNN_WIDTHS[0], CNN_WIDTHS[0]], CNN_WIDTHS[0]
        for i, w in enumerate(CNN_WIDTHS):
            for j in range(2):
                sizes += [w * cin * 9, w, w, w * w * 9, w, w]
                if i > 0 and j == 0:
                    sizes += [w * cin, w, w]
                cin = w
        sizes += [cin * CNN_CLASSES, CNN_CLASSES]
        return [(n, case["dtype"]) for n in sizes]
    rng = random.Random(case["shapes"])
    parts = [math.exp(rng.uniform(0.0, 9.0)) for _ in range(case["count"])]
    sizes = [max(1, int(case["total"] * p / sum(parts))) for p in parts]
    names = ("fp32", "bf16") if case["dtype"] == "mixed" else (case["dtype"],)
    return [(n, rng.choice(names)) for n in sizes]


def work(case):
    if case["op"] == "xent":
        t, d, v, s = case["tokens"], case["features"], case["classes"], SIZES[case["dtype"]]
        train = case["mode"] != "loss"
        return {"bytes": (t * d + v * d) * s * (2 if train else 1) + 8 * t, "flops": (6 if train else 2) * t * d * v}
    if case["op"] == "gn":
        n = case["batch"] * case["height"] * case["width"] * case["channels"]
        # x read and y written; the backward pass reads x and dy and writes dx
        return {"bytes": n * SIZES[case["dtype"]] * (2 if case["mode"] == "infer" else 5),
                "flops": n * (8 if case["mode"] == "infer" else 24)}
    n = sum(k * SIZES[t] for k, t in _clip_shapes(case))
    return {"bytes": 2 * n, "flops": 3 * sum(k for k, _ in _clip_shapes(case))}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _kink(z):
    return z.abs() < 1e-4


def prepare(case, seed):
    g, dev = _generator(seed), _device()
    if case["op"] == "xent":
        t, d, v, dt = case["tokens"], case["features"], case["classes"], DTYPES[case["dtype"]]
        x = torch.randn(t, d, generator=g, device=dev)                         # a final norm's output
        w = torch.randn((v, d) if case["w_is_cd"] else (d, v), generator=g, device=dev).mul_(1.5 / math.sqrt(d))
        labels = torch.randint(0, v, (t,), generator=g, device=dev)
        if t > 1:                                                              # padding, prompts
            labels[torch.rand(t, generator=g, device=dev) < 0.1] = IGNORE
        rows = torch.rand(t, generator=g, device=dev) / t
        return {"case": case, "x": x.to(dt), "w": w.to(dt), "labels": labels, "rows": rows}
    if case["op"] == "gn":
        b, h, w, c, dt = case["batch"], case["height"], case["width"], case["channels"], DTYPES[case["dtype"]]
        x = torch.randn(b, h, w, c, generator=g, device=dev)
        x.mul_(torch.rand(c, generator=g, device=dev) + 0.5).add_(torch.randn(c, generator=g, device=dev) * 0.5)
        x = x.to(dt)
        gamma = (torch.rand(c, generator=g, device=dev) + 0.5).to(DTYPES[case["param"]])
        beta = (torch.randn(c, generator=g, device=dev) * 0.3).to(DTYPES[case["param"]])
        if case["act"] == "relu" and case["mode"] == "train":
            # on ReLU's kink one rounding decides about a whole gradient element: inputs stay clear of it
            _, z = _gn_plain_z(x, gamma, beta, case["groups"])[:2]
            x = torch.where(_kink(z), x.float() + 0.03, x.float()).to(dt)
        dy = (torch.randn(b, h, w, c, generator=g, device=dev) * 1e-2).to(dt) if case["mode"] == "train" else None
        return {"case": case, "x": x, "gamma": gamma, "beta": beta, "dy": dy}
    grads = []
    for n, t in _clip_shapes(case):
        scale = 10.0 ** (torch.rand(1, generator=g, device=dev) * 2 - 3)       # layers differ in size by 100
        grads.append((torch.randn(n, generator=g, device=dev) * scale).to(DTYPES[t]))
    out = [torch.empty_like(a) for a in grads]
    return {"case": case, "grads": grads, "out": out, "max_norm": 1.0 if case["norm"] == "2" else 1e-2}


# ---- plain forms -----------------------------------------------------------------------------------------------

def _xent_plain(s):
    case, labels = s["case"], s["labels"]
    x, w = s["x"].float(), s["w"].float()
    w = w if case["w_is_cd"] else w.t()                                        # [V, D]
    z = x @ w.t()
    top = z.max(1, keepdim=True).values
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    kept = labels != IGNORE
    at = torch.where(kept, labels, 0)
    loss = torch.where(kept, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    del z
    n = kept.sum()
    if case["mode"] == "loss":
        return {"loss": loss.sum() / n, "lse": lse}
    rows = torch.where(kept, s["rows"] if case["mode"] == "rows" else 1.0 / n, 0.0)
    p.mul_(rows[:, None] / total)
    p.scatter_add_(1, at[:, None], -rows[:, None])
    dw = p.t() @ x if case["w_is_cd"] else x.t() @ p
    return {"loss": loss if case["mode"] == "rows" else loss.sum() / n, "lse": lse,
            "dx": (p @ w).to(s["x"].dtype), "dw": dw.to(s["w"].dtype)}


def _gn_plain_z(x, gamma, beta, groups):
    b, h, w, c = x.shape
    v = x.float().view(b, h * w, groups, c // groups)
    mean = v.mean((1, 3), keepdim=True)
    rstd = torch.rsqrt((v - mean).square().mean((1, 3), keepdim=True) + EPS)
    xhat = ((v - mean) * rstd).view(b, h, w, c)
    return xhat, xhat * gamma.float() + beta.float(), mean, rstd


def _gn_plain(s):
    case, x = s["case"], s["x"]
    b, h, w, c = x.shape
    groups, act = case["groups"], case["act"]
    xhat, z, mean, rstd = _gn_plain_z(x, s["gamma"], s["beta"], groups)
    if act == "relu":
        y, slope = z.clamp_min(0), (z > 0).float()
    elif act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        y = z * sig
        slope = sig * (1.0 + z * (1.0 - sig))
    else:
        y, slope = z, 1.0
    got = {"y": y.to(x.dtype), "mean": mean.view(b, groups), "rstd": rstd.view(b, groups)}
    if case["mode"] == "infer":
        return got
    dz = s["dy"].float() * slope
    dxhat = (dz * s["gamma"].float()).view(b, h * w, groups, c // groups)
    xg = xhat.view(b, h * w, groups, c // groups)
    s1, s2 = dxhat.mean((1, 3), keepdim=True), (dxhat * xg).mean((1, 3), keepdim=True)
    dx = ((dxhat - s1 - xg * s2) * rstd).view(b, h, w, c)
    return {**got, "dx": dx.to(x.dtype), "dgamma": (dz * xhat).sum((0, 1, 2)).to(s["gamma"].dtype),
            "dbeta": dz.sum((0, 1, 2)).to(s["beta"].dtype)}


def _clip_plain(s):
    grads = s["grads"]
    if s["case"]["norm"] == "inf":
        norm = torch.stack([a.abs().max().float() for a in grads]).max()
    else:
        norm = torch.sqrt(torch.stack([a.float().square().sum() for a in grads]).sum())
    scale = torch.clamp_max(s["max_norm"] / (norm + CLIP_EPS), 1.0)
    return {"norm": norm, "grads": [(a.float() * scale).to(a.dtype) for a in grads]}


# ---- the library -----------------------------------------------------------------------------------------------

def _xent_own(s):
    from paper_2310_03675_b200 import hdqt
    case, x, w, labels = s["case"], s["x"], s["w"], s["labels"]
    how = {"ignore_index": IGNORE, "w_is_cd": case["w_is_cd"]}
    if case["mode"] == "loss":
        loss, lse = hdqt.linear_xent_fwd(x, w, labels, reduction="mean", **how)
        return {"loss": loss, "lse": lse}
    if case["mode"] == "rows":
        loss, lse = hdqt.linear_xent_fwd(x, w, labels, reduction="none", **how)
        dx, dw = hdqt.linear_xent_bwd(x, w, labels, lse, s["rows"], reduction="none", **how)
    else:
        loss, lse, dx, dw = hdqt.linear_xent_train(x, w, labels, reduction="mean", **how)
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def _gn_own(s):
    from paper_2310_03675_b200 import hdqt
    case = s["case"]
    y, mean, rstd = hdqt.group_norm_fwd(s["x"], s["gamma"], s["beta"], case["groups"], eps=EPS, act=case["act"])
    got = {"y": y, "mean": mean, "rstd": rstd}
    if case["mode"] == "train":
        dx, dgamma, dbeta = hdqt.group_norm_bwd(s["dy"], s["x"], s["gamma"], s["beta"], mean, rstd, case["groups"],
                                                act=case["act"])
        got.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    return got


def _clip_own(s):
    from paper_2310_03675_b200 import hdqt
    norm = hdqt.clip_grad_norm(s["grads"], s["max_norm"], norm_type=float(s["case"]["norm"]), out=s["out"])
    return {"norm": norm, "grads": s["out"]}


def run(state):
    op = state["case"]["op"]
    if own:
        got = {"xent": _xent_own, "gn": _gn_own, "clip": _clip_own}[op](state)
    else:
        got = {"xent": _xent_plain, "gn": _gn_plain, "clip": _clip_plain}[op](state)
    return got


# ---- 64 bits ---------------------------------------------------------------------------------------------------

def _xent_exact(s):
    case = s["case"]
    x, w, labels = s["x"].double(), s["w"].double(), s["labels"]
    if not case["w_is_cd"]:
        w = w.t().contiguous()
    t, v = x.shape[0], w.shape[0]
    kept = labels != IGNORE
    n = int(kept.sum())
    scale = s["rows"].double() if case["mode"] == "rows" else torch.full((t,), 1.0 / n if n else math.nan, device=x.device,
                                                                         dtype=torch.float64)
    lse, loss = torch.empty(t, device=x.device, dtype=torch.float64), torch.zeros(t, device=x.device, dtype=torch.float64)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    step = max(1, (1 << 28) // v)
    for a in range(0, t, step):                       # a few rows at a time
        rows = torch.arange(a, min(t, a + step), device=x.device)
        z = torch.einsum("td,vd->tv", x[rows], w)
        lse[rows] = torch.logsumexp(z, 1)
        own_rows = rows[kept[rows]]
        loss[own_rows] = lse[own_rows] - z[own_rows - a, labels[own_rows]]
        if case["mode"] == "loss":
            continue
        dz = torch.softmax(z, 1)
        dz[own_rows - a, labels[own_rows]] -= 1.0
        dz *= (scale[rows] * kept[rows])[:, None]
        dx[rows] = dz @ w
        dw += torch.einsum("tv,td->vd", dz, x[rows])
    total = loss if case["mode"] == "rows" else loss.sum() / n if n else torch.tensor(math.nan, device=x.device)
    if case["mode"] == "loss":
        return {"loss": total, "lse": lse}
    return {"loss": total, "lse": lse, "dx": dx, "dw": dw if case["w_is_cd"] else dw.t()}


def _gn_exact(s):
    case = s["case"]
    groups, act = case["groups"], case["act"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    per = gamma.numel() // groups
    got = {k: [] for k in ("y", "mean", "rstd", "dx")}
    dgamma, dbeta = torch.zeros_like(gamma), torch.zeros_like(beta)
    for i in range(s["x"].shape[0]):                  # one image at a time
        x = s["x"][i].double().flatten(0, 1)                                   # [pixels, C]
        by_group = x.unflatten(1, (groups, per)).transpose(0, 1).flatten(1)    # [G, pixels * per]
        var, mean = torch.var_mean(by_group, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        spread = lambda v: v.repeat_interleave(per)  # noqa: E731
        xhat = (x - spread(mean)) * spread(rstd)
        z = xhat * gamma + beta
        y = torch.relu(z) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z
        got["y"].append(y.view_as(s["x"][i]))
        got["mean"].append(mean)
        got["rstd"].append(rstd)
        if case["mode"] == "infer":
            continue
        dz = s["dy"][i].double().flatten(0, 1)
        if act == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif act == "silu":
            sig = torch.sigmoid(z)
            dz = dz * (sig + y * (1 - sig))
        dgamma += (dz * xhat).sum(0)
        dbeta += dz.sum(0)
        d = dz * gamma
        over = lambda v: spread(v.sum(0).view(groups, per).mean(1) / x.shape[0])  # noqa: E731
        got["dx"].append(((d - over(d) - xhat * over(d * xhat)) * spread(rstd)).view_as(s["x"][i]))
    out = {k: torch.stack(v) for k, v in got.items() if v}
    return {**out, "dgamma": dgamma, "dbeta": dbeta} if case["mode"] == "train" else out


def _clip_exact(s):
    if s["case"]["norm"] == "inf":
        norm = max(float(a.double().abs().max()) for a in s["grads"])
    else:
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(a.double())) ** 2 for a in s["grads"]))
    scale = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
    return {"norm": norm, "grads": [a.double() * scale for a in s["grads"]]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"xent": _xent_exact, "gn": _gn_exact, "clip": _clip_exact}[case["op"]](s)
