"""Cases of the operators around the residual stream of a network of quantized products, with their plain forms:

  ln    layer norm with an activation over the features of a row, forward and backward
  drop  dropout from the counter-based generator, added to a residual or not, forward and backward
  dal   dropout, residual add and layer norm as one operator, forward and backward

`run` computes the plain form (elementary torch operations in 32 bits, rounded once at the end) while `own` is
false, and calls the library while it is true.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5        # of the layer norm's variance
TAG = 6           # of the dropout's random stream
MASK32 = 0xFFFFFFFF


def _device():
    return torch.device("cuda", torch.cuda.current_device())


def _generator(seed):
    g = torch.Generator(device=_device())
    g.manual_seed(seed)
    return g


# ---- cases -----------------------------------------------------------------------------------------------------

def listed():
    return [
        # hidden layer of the sensor-window network on its batch: a call that is all latency
        {"name": "ln_mlp", "op": "ln", "mode": "train", "rows": 256, "channels": 512, "dtype": "fp32", "param": "fp32",
         "act": "relu"},
        # one token on its way through a model: one row
        {"name": "ln_one_row", "op": "ln", "mode": "infer", "rows": 1, "channels": 4096, "dtype": "bf16",
         "param": "bf16", "act": "none"},
        # ragged batch, odd number of features
        {"name": "ln_odd", "op": "ln", "mode": "train", "rows": 5003, "channels": 1531, "dtype": "fp16", "param": "fp32",
         "act": "silu"},
        # many short rows: a norm per group of features or per patch
        {"name": "ln_narrow", "op": "ln", "mode": "train", "rows": 200000, "channels": 96, "dtype": "fp32",
         "param": "fp32", "act": "none"},
        # an ordinary training micro-batch
        {"name": "ln_mid", "op": "ln", "mode": "train", "rows": 4096, "channels": 2048, "dtype": "bf16", "param": "fp32",
         "act": "none"},
        # the largest: a long batch of wide rows
        {"name": "ln_large", "op": "ln", "mode": "train", "rows": 32768, "channels": 8192, "dtype": "bf16",
         "param": "fp32", "act": "none"},
        # dropout behind a hidden layer of the sensor-window network
        {"name": "drop_mlp", "op": "drop", "rows": 256, "channels": 512, "dtype": "fp32", "p": 0.1, "residual": False},
        # odd sizes, added to a residual
        {"name": "drop_odd", "op": "drop", "rows": 12347, "channels": 777, "dtype": "fp16", "p": 0.25, "residual": True},
        # a large batch of activations
        {"name": "drop_large", "op": "drop", "rows": 32768, "channels": 4096, "dtype": "bf16", "p": 0.1,
         "residual": True},
        # end of a residual block of the sensor-window network: dropout, add, norm, activation
        {"name": "dal_mlp", "op": "dal", "mode": "train", "rows": 256, "channels": 512, "dtype": "fp32", "param": "fp32",
         "act": "relu", "p": 0.1, "stream": False},
        # odd sizes in 16 bits, the sum itself used further on (its gradient arrives too)
        {"name": "dal_odd", "op": "dal", "mode": "train", "rows": 4111, "channels": 1001, "dtype": "bf16",
         "param": "fp32", "act": "none", "p": 0.25, "stream": True},
        # a training micro-batch of a wide residual network
        {"name": "dal_large", "op": "dal", "mode": "train", "rows": 16384, "channels": 4096, "dtype": "bf16",
         "param": "fp32", "act": "none", "p": 0.1, "stream": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("ln", "ln", "drop", "dal", "dal"))
    dtype = rng.choice(("fp32", "bf16", "bf16", "fp16"))
    most = 1 << {"ln": 29, "drop": 28, "dal": 27}[op]          # bytes of one tensor
    while True:
        rows, c = _log_int(rng, 1, 262144), _log_int(rng, 8, 16384)
        if rng.random() < 0.6:                                 # most models keep multiples of 8; the rest is any number
            c = -(-c // 8) * 8
        if rows * c * SIZES[dtype] <= most:
            break
    case = {"op": op, "rows": rows, "channels": c, "dtype": dtype}
    if op != "drop":
        case.update(mode=rng.choice(("train", "train", "infer")), param=rng.choice(("fp32", "fp32", dtype)),
                    act=rng.choice(("none", "none", "relu", "silu")))
    if op != "ln":
        case["p"] = rng.choice((0.1, 0.5, round(rng.uniform(0.01, 0.9), 3)))
    if op == "drop":
        case["residual"] = rng.random() < 0.6
    if op == "dal":
        case["stream"] = case["mode"] == "train" and rng.random() < 0.6
        if case["mode"] == "infer":
            case["p"] = 0.0                                    # no dropout outside training
    return case


def work(case):
    n, s, op = case["rows"] * case["channels"], SIZES[case["dtype"]], case["op"]
    if op == "drop":          # x (and residual) read, y written; dy read, dx written
        return {"bytes": n * s * (5 if case["residual"] else 4), "flops": n * 3}
    train = case["mode"] == "train"
    if op == "ln":            # x read, y written; x and dy read, dx written
        return {"bytes": n * s * (5 if train else 2), "flops": n * (24 if train else 8)}
    # x and residual read, the sum and y written; dy, the sum (and its gradient) read, two gradients written
    return {"bytes": n * s * (4 + (4 + case["stream"] if train else 0)), "flops": n * (28 if train else 10)}


# ---- inputs ----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g, dev, dt, op = _generator(seed), _device(), DTYPES[case["dtype"]], case["op"]
    shape = (case["rows"], case["channels"])

    def normal(scale=1.0):
        return torch.randn(shape, generator=g, device=dev).mul_(scale)

    s = {"case": case, "x": normal()}
    if op == "ln":
        c = case["channels"]
        s["x"].mul_(torch.rand(c, generator=g, device=dev) + 0.5).add_(torch.randn(c, generator=g, device=dev) * 0.5)
    s["x"] = s["x"].to(dt)
    if op != "ln":
        s["seed"] = int(torch.randint(0, 1 << 62, (1,), generator=g, device=dev))
        # a device word that a recorded training step advances
        s["offset"] = torch.randint(0, 1 << 20, (1,), generator=g, device=dev, dtype=torch.int32)
    if op == "drop":
        s["residual"] = normal().to(dt) if case["residual"] else None
        s["dy"] = normal(1e-2).to(dt)
        return s
    c = case["channels"]
    s["gamma"] = (torch.rand(c, generator=g, device=dev) + 0.5).to(DTYPES[case["param"]])
    s["beta"] = (torch.randn(c, generator=g, device=dev) * 0.3).to(DTYPES[case["param"]])
    if op == "dal":
        s["residual"] = normal(2.0).to(dt)
    if case["mode"] == "train":
        if case["act"] == "relu":
            # on ReLU's kink one rounding decides about a whole gradient element: inputs stay clear of it
            side = "x" if op == "ln" else "residual"
            h = s["x"] if op == "ln" else _sum_plain(s, _kept_plain(s))
            z = _norm_plain(h, s["gamma"], s["beta"])[1]
            s[side] = torch.where(z.abs() < 1e-3, s[side].float() + 0.05, s[side].float()).to(dt)
            del h, z
        s["dy"] = normal(1e-2).to(dt)
        s["dh"] = normal(1e-2).to(dt) if case.get("stream") else None
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------

def _philox_plain(groups, seed, tag, offset):
    """Philox4x32-10 of the counters (group, 0 above 32 bits, tag, offset): four words per group, int64 [groups, 4].  The
    low 64 bits of a product are those of the unsigned one, so the words come out by shifting and masking."""
    idx = torch.arange(groups, device=offset.device)
    c = [idx & MASK32, idx >> 32, torch.full_like(idx, tag), (offset.long() & MASK32).expand(groups)]
    k0, k1 = seed & MASK32, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & MASK32) ^ c[1] ^ k0, b & MASK32, ((a >> 32) & MASK32) ^ c[3] ^ k1, a & MASK32]
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    return torch.stack(c, 1)


def _threshold(p):
    """16-bit numbers below it drop their element, and what a kept one is multiplied by."""
    t = round(p * 65536)
    return t, (65536 / (65536 - t) if t < 65536 else 0.0)


def _kept_plain(s):
    case = s["case"]
    n = case["rows"] * case["channels"]
    words = _philox_plain((n + 7) // 8, s["seed"], TAG, s["offset"])
    u = torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:n]            # low half first
    return (u >= _threshold(case["p"])[0]).view(case["rows"], case["channels"])


def _drop_plain(v, kept, p):
    return torch.where(kept, v * torch.tensor(_threshold(p)[1], dtype=torch.float32, device=v.device), 0.0)


def _sum_plain(s, kept):
    """The residual stream as it is held: rounded to its type."""
    x = s["x"].float()
    d = x if kept is None else _drop_plain(x, kept, s["case"]["p"])
    return (d if s["residual"] is None else s["residual"].float() + d).to(s["x"].dtype)


def _norm_plain(x, gamma, beta):
    v = x.float()
    mean = v.mean(1, keepdim=True)
    rstd = torch.rsqrt((v - mean).square().mean(1, keepdim=True) + EPS)
    xhat = (v - mean) * rstd
    return xhat, xhat * gamma.float() + beta.float(), mean, rstd


def _act_plain(z, act):
    if act == "relu":
        return z.clamp_min(0), (z > 0).float()
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return z * sig, sig * (1.0 + z * (1.0 - sig))
    return z, None


def _norm_grad_plain(s, xhat, slope, rstd):
    """Gradient of the norm's input in 32 bits, dgamma and dbeta."""
    dz = s["dy"].float() if slope is None else s["dy"].float() * slope
    d = dz * s["gamma"].float()
    s1, s2 = d.mean(1, keepdim=True), (d * xhat).mean(1, keepdim=True)
    return ((d - s1 - xhat * s2) * rstd, (dz * xhat).sum(0).to(s["gamma"].dtype), dz.sum(0).to(s["beta"].dtype))


def _ln_plain(s):
    case, x = s["case"], s["x"]
    xhat, z, mean, rstd = _norm_plain(x, s["gamma"], s["beta"])
    y, slope = _act_plain(z, case["act"])
    got = {"y": y.to(x.dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    del y, z
    if case["mode"] == "train":
        dx, dgamma, dbeta = _norm_grad_plain(s, xhat, slope, rstd)
        got.update(dx=dx.to(x.dtype), dgamma=dgamma, dbeta=dbeta)
    return got


def _drop_run_plain(s):
    kept = _kept_plain(s)
    dx = _drop_plain(s["dy"].float(), kept, s["case"]["p"])
    return {"y": _sum_plain(s, kept), "dx": dx.to(s["x"].dtype)}


def _dal_plain(s):
    case, dt = s["case"], s["x"].dtype
    kept = _kept_plain(s) if case["p"] > 0 else None
    h = _sum_plain(s, kept)
    xhat, z, mean, rstd = _norm_plain(h, s["gamma"], s["beta"])
    y, slope = _act_plain(z, case["act"])
    got = {"h": h, "y": y.to(dt), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if case["mode"] == "infer":
        return got
    g, dgamma, dbeta = _norm_grad_plain(s, xhat, slope, rstd)
    if s["dh"] is not None:
        g = g + s["dh"].float()
    return {**got, "dx": _drop_plain(g, kept, case["p"]).to(dt), "dresidual": g.to(dt), "dgamma": dgamma, "dbeta": dbeta}


# ---- the library -----------------------------------------------------------------------------------------------

def _ln_own(s):
    from paper_2310_03675_b200 import hdqt
    act = s["case"]["act"]
    y, mean, rstd = hdqt.layer_norm_fwd(s["x"], s["gamma"], s["beta"], eps=EPS, act=act)
    got = {"y": y, "mean": mean, "rstd": rstd}
    if s["case"]["mode"] == "train":
        dx, dgamma, dbeta = hdqt.layer_norm_bwd(s["dy"], s["x"], s["gamma"], s["beta"], mean, rstd, act=act)
        got.update(dx=dx, dgamma=dgamma, dbeta=dbeta)
    return got


def _drop_own(s):
    from paper_2310_03675_b200 import hdqt
    how = {"tag": TAG, "philox_offset": s["offset"]}
    y = hdqt.dropout(s["x"], s["case"]["p"], s["seed"], residual=s["residual"], **how)
    return {"y": y, "dx": hdqt.dropout(s["dy"], s["case"]["p"], s["seed"], **how)}


def _dal_own(s):
    from paper_2310_03675_b200 import hdqt
    case = s["case"]
    how = {"p": case["p"], "seed": s["seed"], "tag": TAG, "philox_offset": s["offset"], "act": case["act"]}
    y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(s["x"], s["residual"], s["gamma"], s["beta"], eps=EPS, **how)
    got = {"h": h, "y": y, "mean": mean, "rstd": rstd}
    if case["mode"] == "train":
        dx, dresidual, dgamma, dbeta = hdqt.dropout_add_layer_norm_bwd(s["dy"], s["dh"], h, s["gamma"], s["beta"], mean,
                                                                       rstd, **how)
        got.update(dx=dx, dresidual=dresidual, dgamma=dgamma, dbeta=dbeta)
    return got


def run(state):
    op = state["case"]["op"]
    if own:
        return {"ln": _ln_own, "drop": _drop_own, "dal": _dal_own}[op](state)
    return {"ln": _ln_plain, "drop": _drop_run_plain, "dal": _dal_plain}[op](state)


# ---- 64 bits ---------------------------------------------------------------------------------------------------

def _mul_hi_lo(a, m):
    """Both 32-bit words of a * m for a < 2^32 and a constant m < 2^32, by halves of m: nothing passes 2^49."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    mid = (low >> 16) + (high & 0xFFFF)                 # weights 2^16
    return (high >> 16) + (mid >> 16), ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _kept_exact(s, first, last):
    """Truth values of the elements first..last - 1 of the flattened tensor."""
    dev = s["x"].device
    group = torch.arange(first // 8, (last + 7) // 8, device=dev)
    x0, x1 = group % (1 << 32), group // (1 << 32)
    x2, x3 = torch.full_like(group, TAG), torch.zeros_like(group) + s["offset"].long()
    for r in range(10):
        key0 = ((s["seed"] % (1 << 32)) + r * 0x9E3779B9) % (1 << 32)
        key1 = ((s["seed"] // (1 << 32)) + r * 0xBB67AE85) % (1 << 32)
        hi0, lo0 = _mul_hi_lo(x0, 0xD2511F53)
        hi1, lo1 = _mul_hi_lo(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = hi1 ^ x1 ^ key0, lo1, hi0 ^ x3 ^ key1, lo0
    at = torch.arange(first, last, device=dev)
    word = torch.stack([x0, x1, x2, x3])[at % 8 // 2, at // 8 - first // 8]
    number = torch.where(at % 2 == 0, word % 65536, word // 65536)
    return number >= round(s["case"]["p"] * 65536)


def exact(case, seed):
    s = prepare(case, seed)
    rows, c, dt, op = case["rows"], case["channels"], s["x"].dtype, case["op"]
    train = op == "drop" or case["mode"] == "train"
    parts, sums = {}, {}
    step = max(1, (1 << 25) // c)

    def put(**tensors):
        for k, v in tensors.items():
            parts.setdefault(k, []).append(v)

    for a in range(0, rows, step):                      # a few rows at a time
        b = min(rows, a + step)
        x = s["x"][a:b].double()
        factor = None                                   # of the dropout
        if op != "ln" and case["p"] > 0:
            drop = round(case["p"] * 65536)
            kept = _kept_exact(s, a * c, b * c).view(b - a, c)
            factor = kept.double() * (65536 / (65536 - drop) if drop < 65536 else 0.0)
            x = x * factor
        if op == "drop":
            put(y=x if s["residual"] is None else x + s["residual"][a:b].double(), dx=s["dy"][a:b].double() * factor)
            continue
        if op == "dal":
            x = x + s["residual"][a:b].double()
            put(h=x)
            x = x.to(dt).double()                       # what is normalised is the sum as it is held
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        rstd = (var + EPS) ** -0.5
        xhat = (x - mean) * rstd
        gamma = s["gamma"].double()
        z = torch.addcmul(s["beta"].double(), xhat, gamma)
        sig = torch.sigmoid(z) if case["act"] == "silu" else None
        put(y=torch.relu(z) if case["act"] == "relu" else z if sig is None else z * sig, mean=mean[:, 0], rstd=rstd[:, 0])
        if not train:
            continue
        dz = s["dy"][a:b].double()
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif sig is not None:
            dz = dz * (sig + z * sig * (1 - sig))
        for k, v in (("dgamma", dz * xhat), ("dbeta", dz)):
            sums[k] = sums.get(k, 0) + v.sum(0)
        d = dz * gamma
        g = rstd * (d - d.sum(1, keepdim=True) / c - xhat * ((d * xhat).sum(1, keepdim=True) / c))
        if op == "ln":
            put(dx=g)
            continue
        if s["dh"] is not None:
            g = g + s["dh"][a:b].double()
        put(dresidual=g, dx=g if factor is None else g * factor)
    return {**{k: torch.cat(v) for k, v in parts.items()}, **sums}
