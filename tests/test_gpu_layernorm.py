"""Layer norm with an activation, alone and behind dropout and a residual add, forward and backward, against 64-bit arithmetic.

Tolerances (e = 2^-24): a row's sums run over at most 41 terms per thread and then over trees of at most 10 additions, so that
a mean of values v is off by at most 52 e mean|v|, a variance by as much of itself (and 1/sqrt by half), and with the roundings around
them, per element,
  xhat off by 96 e rs (mean|x| + |x|),  z by |gamma| times that plus a few e (|beta| + |z|)
  SiLU adds 2^-20 |z| (fast exponential: 2 units of 2^-22 plus |z| e), its derivative 2^-19
  dx   the same errors through its three terms, the two means of gamma dz and gamma dz xhat off by 192 e of the mean magnitude
  dgamma, dbeta: at most 512 terms one after the other, 512 e sum|term|
and every output is rounded once to its type (e, 2^-8, 2^-11).
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import hdqt_oracle as O
from paper_2310_03675_b200 import hdqt

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a unit in the last place
E = 2.0 ** -24
EPS = 1e-5


def reference(x, gamma, beta, act, dy=None, dh=None, eps=EPS, terms=96):
    """64-bit forward and backward over the last dimension, with the error bounds of the docstring (`terms` in the place of 96)."""
    c = x.shape[-1]
    xd = x.double()
    g = torch.ones(c, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(c, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    mean = lambda t: t.mean(-1, keepdim=True)  # noqa: E731
    mu = mean(xd)
    rs = (mean((xd - mu) ** 2) + eps) ** -0.5
    xh = (xd - mu) * rs
    z = xh * g + b
    size = mean(xd.abs()) + xd.abs()
    exh = terms * E * rs * size
    ez = g.abs() * exh + 8 * E * (b.abs() + z.abs())
    sig = torch.sigmoid(z)
    y = {"none": z, "relu": z.clamp_min(0), "silu": z * sig}[act]
    out = {"y": (y, ez * 1.2 + (2.0 ** -20 * z.abs() if act == "silu" else 0)),
           "mean": (mu[..., 0], terms * E * mean(xd.abs())[..., 0]),
           "rstd": (rs[..., 0], (rs * terms * E * (1 + rs * mean(xd.abs())))[..., 0]),
           "z_margin": float((z.abs() / (ez + 1e-30)).min()) if z.numel() else 2.0}
    if dy is not None:
        d = dy.double()
        slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": sig * (1 + z * (1 - sig))}[act]
        eslope = {"none": 0.0, "relu": 0.0, "silu": 2.0 ** -19 + 0.5 * ez}[act]
        dz, edz = d * slope, d.abs() * (eslope + 4 * E)
        dg, edg = dz * g, edz * g.abs()
        m1, m2 = mean(dg), mean(dg * xh)
        em1 = mean(edg) + 2 * terms * E * mean(dg.abs())
        em2 = mean(edg * xh.abs() + dg.abs() * exh) + 2 * terms * E * mean((dg * xh).abs())
        dx = rs * (dg - m1 - xh * m2)
        edx = rs * (edg + em1 + xh.abs() * em2 + exh * m2.abs() + 16 * E * (dg.abs() + m1.abs() + (xh * m2).abs())) + dx.abs() * 128 * E
        if dh is not None:
            dx = dx + dh.double()
            edx = edx + E * dx.abs()
        out["dx"] = (dx, edx)
        total = lambda t: t.reshape(-1, c).sum(0)  # noqa: E731
        out["dgamma"] = (total(dz * xh), total(edz * xh.abs() + dz.abs() * exh) + 512 * E * total((dz * xh).abs()))
        out["dbeta"] = (total(dz), total(edz) + 512 * E * total(dz.abs()))
    return out


def close(got, want):
    value, err = want
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 1e-37
    good = (got.double() - value).abs() <= err + UNIT[got.dtype] * (value.abs() + err) + tiny
    assert bool(good.all()), (int((~good).sum()), float(((got.double() - value).abs() / (err + UNIT[got.dtype] * value.abs() + tiny)).max()))


def inputs(shape, dtype, param, seed, offset=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = shape[-1]
    x = torch.randn(shape, generator=g, device="cuda") * (torch.rand(c, generator=g, device="cuda") + 0.5)
    x = (x + offset * torch.randn(c, generator=g, device="cuda")).to(DT[dtype])
    gamma = (torch.rand(c, generator=g, device="cuda") + 0.5).to(DT[param])
    beta = (0.3 * torch.randn(c, generator=g, device="cuda")).to(DT[param])
    dy = (0.1 * torch.randn(shape, generator=g, device="cuda")).to(DT[dtype])
    return x, gamma, beta, dy


def away_from_kink(x, gamma, beta):
    """ReLU's derivative jumps at 0: moves the few inputs whose z is within the error of one rounding of it."""
    z = reference(x, gamma, beta, "none")["y"][0]
    return torch.where(z.abs() < 1e-3, x.float() + 0.05, x.float()).to(x.dtype)


def kept(n, p, seed, tag=0, offset=0):
    """Which of n elements stay, from the oracle's generator."""
    g = np.arange((n + 7) // 8, dtype=np.uint64)
    w = O.philox4x32_10(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.full_like(g, tag), np.full_like(g, offset),
                        seed & 0xFFFFFFFF, seed >> 32)
    w = np.stack([np.asarray(v, dtype=np.uint64) for v in w], 1)
    u = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[:n]
    return torch.from_numpy((u >= np.uint64(round(p * 65536))))


def scale_of(p):
    t = round(p * 65536)
    return np.float32(65536 / (65536 - t)) if t < 65536 else np.float32(0)


SHAPES = [
    (40,), (1, 1), (3, 1), (1, 8), (5, 7), (2, 33), (37, 30), (3, 4, 12), (1000, 64), (130, 96), (17, 257), (33, 512), (9, 1000),
    (4, 1024), (5, 1531), (1500, 1152), (7, 2048), (300, 2050), (3, 4096), (2, 4100), (700, 4104), (2, 8192), (3, 8200), (2, 10001),
    (3, 7999), (2, 8000), (2, 8191), (2, 16384), (1, 16390), (2, 33000), (2, 40001),
    # enough rows for teams that walk over several
    (3001, 7), (5000, 24), (2003, 90), (1999, 128), (1700, 256), (1501, 260), (1203, 513), (901, 1001), (700, 1531), (610, 3001), (450, 6001),
    (401, 8200), (351, 10001), (330, 16384), (300, 16383), (296, 777), (297, 1000),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,param", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward_match_64_bits(shape, dtype, param):
    for act in ("none", "relu", "silu"):
        x, gamma, beta, dy = inputs(shape, dtype, param, seed=shape[-1])
        if act == "relu":
            x = away_from_kink(x, gamma, beta)
        want = reference(x, gamma, beta, act, dy)
        y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS, act)
        for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
            close(got, want[name])
        if act == "relu" and want["z_margin"] < 1:
            continue      # an input on the kink after all
        dx, dgamma, dbeta = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd, act)
        for got, name in ((dx, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
            close(got, want[name])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,param", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_fused_with_dropout_and_residual(shape, dtype, param):
    n = math.prod(shape)
    seed, tag = 0x1234567890ABCDEF, 14
    offset = torch.tensor([77], dtype=torch.int32, device="cuda")
    for act, p, with_res, with_dh in (("none", 0.25, True, True), ("silu", 0.1, False, False), ("none", 0.0, True, True)):
        x, gamma, beta, dy = inputs(shape, dtype, param, seed=shape[-1] + 1)
        res, _, _, dh = inputs(shape, dtype, param, seed=shape[-1] + 2)
        res, dh = res if with_res else None, dh if with_dh else None
        how = dict(p=p, seed=seed, tag=tag, philox_offset=offset, act=act)
        keep = kept(n, p, seed, tag, 77).cuda().view(shape)
        factor = torch.where(keep, torch.tensor(scale_of(p), device="cuda"), 0.0)
        y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x, res, gamma, beta, eps=EPS, **how)
        dropped = torch.where(keep, x.float() * torch.tensor(scale_of(p), device="cuda"), 0.0)
        assert torch.equal(h, (dropped if res is None else res.float() + dropped).to(x.dtype))
        want = reference(h, gamma, beta, act, dy, dh)
        for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
            close(got, want[name])
        dx, dres, dgamma, dbeta = hdqt.dropout_add_layer_norm_bwd(dy, dh, h, gamma, beta, mean, rstd, **how)
        for got, name in ((dres, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
            close(got, want[name])
        f = factor.double()
        close(dx, (want["dx"][0] * f, want["dx"][1] * f + E * (want["dx"][0] * f).abs()))
        assert not bool(dx[~keep].any())
        # the parts are the same whatever else is asked for, and h that of the two operators one after the other
        some = hdqt.dropout_add_layer_norm_bwd(dy, dh, h, gamma, beta, mean, rstd, want_residual=False, want_params=False, **how)
        assert torch.equal(some[0], dx) and some[1] is None and some[2] is None
        two = hdqt.dropout(x, p, seed, tag, res, offset)
        assert torch.equal(two, h)
        y2, mean2, rstd2 = hdqt.layer_norm_fwd(two, gamma, beta, EPS, act)
        for got, name in ((y2, "y"), (mean2, "mean"), (rstd2, "rstd")):      # (a row may be divided otherwise: sums in another order)
            close(got, want[name])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_slices_odd_addresses_and_missing_parameters(dtype):
    wide, gamma, beta, dy = inputs((6, 7, 96), dtype, "fp32", seed=1)
    for lo, hi in ((0, 16), (8, 24), (3, 21), (47, 48), (2, 96), (1, 95)):
        x, d, r = wide[..., lo:hi], dy[..., lo:hi], wide.flip(0)[..., lo:hi]
        for g, b in ((None, None), (gamma[lo:hi], None), (None, beta[lo:hi]), (gamma[lo:hi], beta[lo:hi])):
            want = reference(x, g, b, "silu", d)
            y, mean, rstd = hdqt.layer_norm_fwd(x, g, b, EPS, "silu")
            assert y.is_contiguous()
            close(y, want["y"])
            dx, dgamma, dbeta = hdqt.layer_norm_bwd(d, x, g, b, mean, rstd, "silu")
            assert (dgamma is None) == (g is None) and (dbeta is None) == (b is None)
            close(dx, want["dx"])
            for got, name in ((dgamma, "dgamma"), (dbeta, "dbeta")):
                if got is not None:
                    close(got, want[name])
        # the random numbers go by the position in the dense tensor, not by the strides
        a = hdqt.dropout_add_layer_norm_fwd(x, r, None, None, 0.5, 3)
        b = hdqt.dropout_add_layer_norm_fwd(x.contiguous(), r.contiguous(), None, None, 0.5, 3)
        assert torch.equal(a[1], b[1])
        if lo % 8 == 0:      # (narrower accesses add in another order)
            assert all(torch.equal(u, v) for u, v in zip(a, b))
    close(hdqt.layer_norm_fwd(wide[::2, 3], gamma, beta, EPS)[0], reference(wide[::2, 3], gamma, beta, "none")["y"])
    with pytest.raises(ValueError):
        hdqt.layer_norm_fwd(wide[:, ::2], gamma, beta)                     # not evenly spaced
    with pytest.raises(ValueError):
        hdqt.layer_norm_fwd(wide[0, :1].expand(4, 96), gamma, beta)        # rows on one another
    with pytest.raises(ValueError):
        hdqt.layer_norm_fwd(wide[0].t(), None, None)                       # channels apart


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("lo,hi", [(8, 104), (16, 72), (0, 200), (1, 34), (3, 200), (5, 101), (64, 65)])
def test_many_rows_of_wider_tensors(dtype, lo, hi):
    """Rows apart in memory, at 16-byte boundaries and elsewhere, more of them than blocks."""
    wide, gamma, beta, dy = inputs((1700, 200), dtype, "fp32", seed=hi)
    other = inputs((1700, 248), dtype, "fp32", seed=hi + 1)[0]
    x, d, r = wide[:, lo:hi], dy[:, lo:hi], other[:, lo:hi]
    g, b = gamma[lo:hi], beta[lo:hi]
    want = reference(x, g, b, "silu", d)
    y, mean, rstd = hdqt.layer_norm_fwd(x, g, b, EPS, "silu")
    for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
        close(got, want[name])
    for got, name in zip(hdqt.layer_norm_bwd(d, x, g, b, mean, rstd, "silu"), ("dx", "dgamma", "dbeta")):
        close(got, want[name])
    y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x, r, g, b, 0.3, 8, eps=EPS)
    keep = kept(h.numel(), 0.3, 8).cuda().view(h.shape)
    assert torch.equal(h, (r.float() + torch.where(keep, x.float() * torch.tensor(scale_of(0.3), device="cuda"), 0.0)).to(x.dtype))
    close(y, reference(h, g, b, "none")["y"])
    # h, dy and dx at addresses that no 16-byte access fits, all in one call
    if hi - lo > 1:
        n = h.numel()
        odd = lambda t: torch.empty(n + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t)  # noqa: E731
        ho, do = odd(h), odd(d)
        want = reference(h, g, b, "none", d)
        dx, dres, dgamma, dbeta = hdqt.dropout_add_layer_norm_bwd(do, None, ho, g, b, mean, rstd, 0.3, 8)
        for got, name in ((dres, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
            close(got, want[name])
        assert not bool(dx[~keep].any()) and torch.equal(dx != 0, keep & (dres != 0))


@pytest.mark.gpu
def test_large_mean_constant_rows_and_outliers():
    x, gamma, beta, dy = inputs((20, 1000), "fp32", "fp32", seed=3)
    x = x + 1000.0
    want = reference(x, gamma, beta, "none", dy)
    y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS)
    close(y, want["y"])
    assert float((rstd.double() / want["rstd"][0] - 1).abs().max()) < 1e-5     # the variance loses no digits to the mean
    for c in (8, 1000, 33000):
        const = torch.full((3, c), 3.0, device="cuda")
        y, mean, rstd = hdqt.layer_norm_fwd(const, None, beta[:8].repeat(c // 8 + 1)[:c].contiguous(), EPS)
        # 41 terms and 10 additions of equal values: the mean is off by at most 52 e, multiplied by 1/sqrt(eps)
        assert float((mean - 3).abs().max()) <= 52 * E * 3
        assert float((y - beta[:8].repeat(c // 8 + 1)[:c]).abs().max()) <= 52 * E * 3 * EPS ** -0.5 + E
    x, gamma, beta, dy = inputs((4, 2048), "fp32", "fp32", seed=4)
    x[:, 0] = 1e4                                                              # one value far out
    want = reference(x, gamma, beta, "none", dy)
    y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS)
    close(y, want["y"])
    close(hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd)[0], want["dx"])


@pytest.mark.gpu
@pytest.mark.parametrize("c", [7, 24, 64, 96, 600, 1001, 4096])
def test_means_above_the_spread_among_others(c):
    """Rows far from zero, constant ones, ones whose squares overflow and ordinary ones, in one call with more rows than blocks; the
    bounds of the docstring hold for each, and no row's result depends on its neighbours."""
    rows = max(3000, 12000000 // c // 8)
    x, gamma, beta, dy = inputs((rows, c), "fp32", "fp32", seed=c)
    plain = x.clone()
    x[1::5] += 1000.0
    x[2::5] = 3.0
    x[3::15] = 3e19 + 1e17 * x[3::15]
    x[4::15] *= 1e-25
    want = reference(x, gamma, beta, "none", dy)
    y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[2::5] = False                          # (a constant row: the rounding of its mean over sqrt(eps), and no more)
    for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
        close(got[keep], tuple(t[keep] for t in want[name]))
    assert float((mean[2::5] - 3).abs().max()) <= 52 * E * 3
    assert float((y[2::5] - beta).abs().max()) <= 1.5 * (52 * E * 3 * EPS ** -0.5 + E)
    dx = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd)[0]
    close(dx[keep], tuple(t[keep] for t in want["dx"]))
    y2, mean2, rstd2 = hdqt.layer_norm_fwd(plain, gamma, beta, EPS)
    assert torch.equal(y[0::5], y2[0::5]) and torch.equal(mean[0::5], mean2[0::5]) and torch.equal(rstd[0::5], rstd2[0::5])
    h = hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, 0.0, 1, eps=EPS)
    close(h[0][keep], tuple(t[keep] for t in want["y"]))


@pytest.mark.gpu
@pytest.mark.parametrize("c", [40, 2024, 4099, 16384])
def test_mean_of_a_few_rows_that_nearly_cancel(c):
    """Summed in 64 bits and rounded once: e |mean|, and 2^-50 of the values' size for the 64-bit sum itself."""
    x = inputs((3, c), "fp32", "fp32", seed=c, offset=0.0)[0]
    x = x - x.mean(1, keepdim=True) + 1e-6
    for mean in (hdqt.layer_norm_fwd(x, None, None, EPS)[1], hdqt.dropout_add_layer_norm_fwd(x, None, None, None, 0.0, 1)[2]):
        want = x.double().mean(1)
        assert bool(((mean.double() - want).abs() <= E * want.abs() + 2.0 ** -50 * x.abs().double().mean(1)).all())


@pytest.mark.gpu
def test_gradients_match_differences():
    """<grad, v> against (L(+h v) - L(-h v)) / 2h with h = 2^-5 and L formed in 64 bits from the call's outputs: the
    third-derivative term is h^2/6 = 1.6e-4 times O(1), the rounding of L e sqrt(n) |y| / h = 1e-4 of |v||c|."""
    x, gamma, beta, dy = inputs((11, 60), "fp32", "fp32", seed=9)
    res, _, _, dh = inputs((11, 60), "fp32", "fp32", seed=10)
    g = torch.Generator(device="cuda").manual_seed(1)
    for act in ("none", "silu"):
        how = dict(p=0.3, seed=5, tag=1, act=act)

        def forward(x, res, gamma, beta):
            return hdqt.dropout_add_layer_norm_fwd(x, res, gamma, beta, eps=EPS, **how)

        y, h, mean, rstd = forward(x, res, gamma, beta)
        grads = hdqt.dropout_add_layer_norm_bwd(dy, dh, h, gamma, beta, mean, rstd, **how)
        for which, grad in enumerate(grads):
            args = [x, res, gamma, beta]
            v = torch.randn(args[which].shape, generator=g, device="cuda")
            step, loss = 2.0 ** -5, []
            for sign in (1, -1):
                moved = list(args)
                moved[which] = args[which] + sign * step * v
                y, h = forward(*moved)[:2]
                loss.append(float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum()))
            want = (loss[0] - loss[1]) / (2 * step)
            scale = float(dy.norm() + dh.norm()) * float(v.norm())
            assert abs(float((grad.double() * v.double()).sum()) - want) <= 1e-3 * scale


@pytest.mark.gpu
def test_non_finite_values_stay_in_their_row():
    for c in (16, 96, 2048, 33000):
        x, gamma, beta, dy = inputs((5, c), "fp32", "fp32", seed=4)
        for value, act in ((math.nan, "silu"), (math.inf, "relu"), (-math.inf, "none")):
            x[3, c // 2] = value
            y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS, act)
            bad = torch.zeros_like(x, dtype=torch.bool)
            bad[3] = True
            assert torch.equal(torch.isnan(y), bad)
            dx, dgamma, dbeta = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd, "none")
            assert torch.equal(torch.isnan(dx), bad) and bool(torch.isnan(dgamma).all()) and bool(torch.isfinite(dbeta).all())
    # dropped elements hold garbage
    x, gamma, beta, _ = inputs((4, 64), "bf16", "fp32", seed=5)
    keep = kept(256, 0.5, 11).cuda().view(4, 64)
    clean = hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, 0.5, 11)
    dirty = hdqt.dropout_add_layer_norm_fwd(torch.where(keep, x, math.nan), None, gamma, beta, 0.5, 11)
    assert all(torch.equal(a, b) for a, b in zip(clean, dirty))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_longest_rows(dtype):
    """2^20 channels: 1024 terms per thread and 10 additions behind them in a sum, so 1100 e in the place of 96 e."""
    x, gamma, beta, dy = inputs((3, 1 << 20), dtype, "fp32", seed=2)
    res = inputs((3, 1 << 20), dtype, "fp32", seed=3)[0]
    want = reference(x, gamma, beta, "none", dy, terms=1100)
    y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS)
    for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
        close(got, want[name])
    for got, name in zip(hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd), ("dx", "dgamma", "dbeta")):
        close(got, want[name])
    y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x, res, gamma, beta, 0.5, 3, eps=EPS)
    want = reference(h, gamma, beta, "none", dy, res, terms=1100)
    close(y, want["y"])
    dx, dres, dgamma, dbeta = hdqt.dropout_add_layer_norm_bwd(dy, res, h, gamma, beta, mean, rstd, 0.5, 3)
    for got, name in ((dres, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
        close(got, want[name])
    assert torch.equal(h, hdqt.dropout(x, 0.5, 3, residual=res))
    assert torch.equal(dx != 0, (hdqt.dropout(torch.ones_like(x), 0.5, 3) != 0) & (dres != 0))


@pytest.mark.gpu
def test_no_rows():
    gamma, beta = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    for shape in ((0, 8), (3, 0, 8)):
        x = torch.empty(shape, device="cuda")
        y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta)
        assert y.shape == x.shape and mean.shape == shape[:-1]
        dx, dgamma, dbeta = hdqt.layer_norm_bwd(x, x, gamma, beta, mean, rstd)
        assert dx.shape == x.shape and not dgamma.any() and not dbeta.any()
        y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x, x, gamma, beta, 0.5, 1)
        out = hdqt.dropout_add_layer_norm_bwd(x, None, h, gamma, beta, mean, rstd, 0.5, 1)
        assert h.shape == y.shape == out[0].shape == out[1].shape and not out[2].any() and not out[3].any()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(700, 96), (300, 1001), (260, 4096), (40, 12000)], ids=str)
def test_parts_repeatability_streams_and_graphs(shape):
    x, gamma, beta, dy = inputs(shape, "bf16", "fp32", seed=5)
    y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta, EPS, "silu")
    dx, dgamma, dbeta = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd, "silu")
    only_dx = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd, "silu", want_params=False)
    only_params = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd, "silu", want_dx=False)
    assert torch.equal(only_dx[0], dx) and only_dx[1] is None and only_params[0] is None
    assert torch.equal(only_params[1], dgamma) and torch.equal(only_params[2], dbeta)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = hdqt.layer_norm_bwd(dy, x, gamma, beta, mean, rstd, "silu")
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))
    # two recorded calls with a workspace each, replayed one after the other, with a device word that advances between replays
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    graphs = []
    for tag in (1, 2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x, dy, gamma, beta, 0.2, 9, tag, philox_offset=word)
            out = hdqt.dropout_add_layer_norm_bwd(dy, None, h, gamma, beta, mean, rstd, 0.2, 9, tag, philox_offset=word)
        graphs.append((graph, (y, h, mean, rstd) + out))
    seen = []
    for k in range(3):
        for tag, (graph, got) in zip((1, 2), graphs):
            graph.replay()
        for tag, (graph, got) in zip((1, 2), graphs):
            y, h, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x, dy, gamma, beta, 0.2, 9, tag, philox_offset=word)
            out = hdqt.dropout_add_layer_norm_bwd(dy, None, h, gamma, beta, mean, rstd, 0.2, 9, tag, philox_offset=word)
            assert all(torch.equal(a, b) for a, b in zip(got, (y, h, mean, rstd) + out))
            seen.append(h)
        word += 1
    assert all(not torch.equal(seen[i], seen[j]) for i in range(6) for j in range(i))


@pytest.mark.gpu
def test_argument_checks():
    x, gamma, beta, dy = inputs((4, 32), "bf16", "fp32", seed=5)
    y, mean, rstd = hdqt.layer_norm_fwd(x, gamma, beta)
    bad = [
        lambda: hdqt.layer_norm_fwd(x.double(), gamma, beta),
        lambda: hdqt.layer_norm_fwd(x, gamma[:31], beta),
        lambda: hdqt.layer_norm_fwd(x, gamma, beta.bfloat16()),
        lambda: hdqt.layer_norm_fwd(x, gamma.half(), beta.half()),
        lambda: hdqt.layer_norm_fwd(x, gamma.cpu(), beta),
        lambda: hdqt.layer_norm_fwd(x, gamma, beta, act="gelu"),
        lambda: hdqt.layer_norm_fwd(x[:, :0], None, None),
        lambda: hdqt.layer_norm_bwd(dy.float(), x, gamma, beta, mean, rstd),
        lambda: hdqt.layer_norm_bwd(dy[:2], x, gamma, beta, mean, rstd),
        lambda: hdqt.layer_norm_bwd(dy, x, gamma, beta, mean[:2], rstd),
        lambda: hdqt.layer_norm_bwd(dy, x, gamma, beta, mean.bfloat16(), rstd),
        lambda: hdqt.layer_norm_bwd(dy, x, gamma, beta, mean.cpu(), rstd),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, dy[:2], gamma, beta, 0.1, 1),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, dy.float(), gamma, beta, 0.1, 1),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, 1.5, 1),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, math.nan, 1),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, 0.1, -1),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, 0.1, 1, tag=1 << 32),
        lambda: hdqt.dropout_add_layer_norm_fwd(x, None, gamma, beta, 0.1, 1, philox_offset=torch.zeros(1, device="cuda")),
        lambda: hdqt.dropout_add_layer_norm_bwd(dy, dy[:1], x, gamma, beta, mean, rstd, 0.1, 1),
        lambda: hdqt.dropout_add_layer_norm_bwd(dy[:, :16], None, x[:, :16], None, None, mean, rstd, 0.1, 1),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} went through")
    with pytest.raises(hdqt.HdqtError):
        hdqt.layer_norm_fwd(x, gamma, beta, eps=-1.0)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """2.2e9 elements: the last rows against 64 bits."""
    rows, c = 2200000, 1000
    x = torch.empty((rows, c), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 200000):
        x[i:i + 200000].normal_(0.5, 1.0)
    y, mean, rstd = hdqt.layer_norm_fwd(x, None, None, EPS, "silu")
    dx, _, _ = hdqt.layer_norm_bwd(x, x, None, None, mean, rstd, "silu", want_params=False)
    for part in (slice(0, 3), slice(rows - 3, rows)):
        want = reference(x[part], None, None, "silu", x[part])
        close(y[part], want["y"])
        close(dx[part], want["dx"])
    del dx
    h = hdqt.dropout_add_layer_norm_fwd(x, None, None, None, 0.5, 3)[1]
    assert torch.equal(h.view(-1), hdqt.dropout(x.view(-1), 0.5, 3))
    assert torch.equal(h[-1] != 0, last_kept(rows * c, c, 0.5, 3).cuda() & (x[-1] != 0))


def last_kept(n, count, p, seed):
    """Which of the last `count` of n elements stay."""
    i = np.arange(n - count, n, dtype=np.uint64)
    g = i // np.uint64(8)
    w = O.philox4x32_10(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.zeros_like(g), np.zeros_like(g), seed, 0)
    w = np.stack([np.asarray(v, dtype=np.uint64) for v in w], 1)
    j = (i % np.uint64(8)).astype(np.int64)
    word = w[np.arange(count), j // 2]
    u = np.where(j % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    return torch.from_numpy(u >= np.uint64(round(p * 65536)))


def test_refusals():
    with pytest.raises(ValueError):
        hdqt.layer_norm_fwd(torch.zeros(2, 8), None, None)                     # not on a GPU
    lib = hdqt.lib
    INVALID, UNSUPPORTED, ALIGN, WS = 1, 2, 3, 4

    def desc(**over):
        d = hdqt.LayerNormDesc(9, 16, 16, 16, 16, 0, 0, 0, 1e-5, 0.5, 7, None, 3, 0)
        for k, v in over.items():
            setattr(d, k, v)
        return d

    def fwd(d, x=256, y=256, gamma=256, mean=256):
        return lib.hdqt_layer_norm_fwd(C.byref(d), x, gamma, 256, y, mean, 256, None)

    def fused(d, x=256, res=256, h=256):
        return lib.hdqt_dropout_add_layer_norm_fwd(C.byref(d), x, res, 256, 256, h, 256, 256, 256, None)

    for bad in ({"channels": 0}, {"channels": -1}, {"rows": -1}, {"dtype": 7}, {"param_dtype": 1}, {"act": 3}, {"act": -1},
                {"eps": -1.0}, {"eps": math.nan}, {"x_row_stride": 15}, {"y_row_stride": 8}):
        assert fwd(desc(**bad)) == INVALID, bad
        assert fused(desc(**bad)) == INVALID, bad
        assert lib.hdqt_layer_norm_workspace_bytes(C.byref(desc(**bad))) == 0
    for bad in ({"p": -0.1}, {"p": 1.1}, {"p": math.nan}, {"r_row_stride": 15}):
        assert fused(desc(**bad)) == INVALID, bad
    assert fwd(desc(channels=1 << 21, x_row_stride=1 << 21, y_row_stride=1 << 21)) == UNSUPPORTED
    assert fwd(desc(rows=1 << 31)) == UNSUPPORTED
    assert fwd(desc(), x=None) == INVALID and fwd(desc(), y=None) == INVALID and fwd(desc(), mean=None) == INVALID
    assert fused(desc(), h=None) == INVALID
    assert fwd(desc(), x=258) == ALIGN and fwd(desc(), gamma=257) == ALIGN and fwd(desc(), mean=258) == ALIGN
    assert fused(desc(), res=258) == ALIGN and fused(desc(), h=257) == ALIGN and fused(desc(philox_offset=258)) == ALIGN
    assert fwd(desc(rows=0), x=None, y=None, mean=None) == 0

    def bwd(d, dy=256, dx=256, ws=256, ws_bytes=1 << 20):
        return lib.hdqt_layer_norm_bwd(C.byref(d), dy, 256, 256, 256, 256, 256, dx, 256, 256, ws, ws_bytes, None)

    many = desc(rows=1000)                                                     # (few rows need no workspace)
    assert lib.hdqt_layer_norm_workspace_bytes(C.byref(desc())) == 0 < lib.hdqt_layer_norm_workspace_bytes(C.byref(many))
    assert bwd(desc(), dy=None) == INVALID and bwd(many, ws=None) == INVALID and bwd(desc(), dx=258) == ALIGN
    assert bwd(many, ws=384 + 8) == ALIGN and bwd(many, ws_bytes=8) == WS
    assert lib.hdqt_dropout_add_layer_norm_bwd(C.byref(desc(p=2.0)), *[256] * 12, 1 << 20, None) == INVALID
    assert lib.hdqt_dropout_add_layer_norm_bwd(C.byref(many), *[256] * 12, 8, None) == WS
    assert lib.hdqt_dropout_add_layer_norm_bwd(C.byref(desc()), 256, 258, *[256] * 10, 1 << 20, None) == ALIGN
