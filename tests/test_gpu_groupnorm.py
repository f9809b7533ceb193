"""Group norm with an activation, forward and backward, against 64-bit arithmetic.

Tolerances (e = 2^-24): sums run over at most 64 terms per thread and then over a tree, so that a mean of values v is off by at most
~96 e mean|v| together with the roundings around it.  So, per element,
  z    off by 96 e (|gamma| rs (mean|x| + |x|) + |beta|)             (x - mu cancels: the error is that of x and mu)
  SiLU adds 2^-20 |z| (fast exponential: 2 units of 2^-22 plus |z| e), its derivative 2^-19
  dx   off by rs |gamma dz|-sized terms x 192 e, plus |x - mu| error through xhat
  dgamma, dbeta: up to 512 terms one after the other, 512 e sum|term|
and every output is rounded once to its type (e, 2^-8, 2^-11).
"""
import math

import pytest
import torch

from paper_2310_03675_b200 import hdqt

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a unit in the last place
E = 2.0 ** -24
EPS = 1e-5


def reference(x, gamma, beta, groups, act, dy=None, eps=EPS):
    """64-bit forward and backward, and the error bounds of the docstring."""
    b, c = x.shape[0], x.shape[-1]
    xd = x.double().reshape(b, -1, groups, c // groups)
    g = torch.ones(c, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    be = torch.zeros(c, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    mu = xd.mean((1, 3), keepdim=True)
    rs = (((xd - mu) ** 2).mean((1, 3), keepdim=True) + eps) ** -0.5
    xh = (xd - mu) * rs
    gg, bb = g.view(1, 1, groups, -1), be.view(1, 1, groups, -1)
    z = xh * gg + bb
    size = xd.abs().mean((1, 3), keepdim=True) + xd.abs()
    exh = 96 * E * rs * size
    ez = gg.abs() * exh + 96 * E * (bb.abs() + z.abs())
    sig = torch.sigmoid(z)
    y = {"none": z, "relu": z.clamp_min(0), "silu": z * sig}[act]
    ey = ez * 1.2 + (2.0 ** -20 * z.abs() if act == "silu" else 0)
    out = {"y": (y.reshape(x.shape), ey.reshape(x.shape)), "mean": (mu.view(b, groups), 96 * E * size.mean((1, 3))),
           "rstd": (rs.view(b, groups), rs.view(b, groups) * (96 * E * (1 + (rs * size.mean((1, 3), keepdim=True)).view(b, groups) ** 1)))}
    out["z_err"] = (z.abs() / (ez + 1e-30)).min()
    if dy is not None:
        d = dy.double().reshape(xd.shape)
        slope = {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": sig * (1 + z * (1 - sig))}[act]
        eslope = {"none": 0.0, "relu": 0.0, "silu": 2.0 ** -19 + 0.5 * ez}[act]
        dz, edz = d * slope, d.abs() * (eslope + 4 * E)
        dg = dz * gg
        m1, m2 = dg.mean((1, 3), keepdim=True), (dg * xh).mean((1, 3), keepdim=True)
        dx = rs * (dg - m1 - xh * m2)
        mean = lambda t: t.mean((1, 3), keepdim=True)  # noqa: E731
        edg = edz * gg.abs()
        em1 = mean(edg) + 192 * E * mean(dg.abs())
        em2 = mean(edg * xh.abs() + dg.abs() * exh) + 192 * E * mean((dg * xh).abs())
        edx = rs * (edg + em1 + xh.abs() * em2 + exh * m2.abs() + 16 * E * (dg.abs() + m1.abs() + (xh * m2).abs())) + dx.abs() * 128 * E
        out["dx"] = (dx.reshape(x.shape), edx.reshape(x.shape))
        sum_c = lambda t: t.sum((0, 1)).reshape(-1)  # noqa: E731
        out["dgamma"] = (sum_c(dz * xh), sum_c(edz * xh.abs() + dz.abs() * exh) + 512 * E * sum_c((dz * xh).abs()))
        out["dbeta"] = (sum_c(dz), sum_c(edz) + 512 * E * sum_c(dz.abs()))
    return out


def close(got, want):
    value, err = want
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 1e-37
    bad = (got.double() - value).abs() > err + UNIT[got.dtype] * (value.abs() + err) + tiny
    assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - value).abs() / (err + UNIT[got.dtype] * value.abs() + tiny)).max()))


def inputs(shape, dtype, param, seed, offset=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = shape[-1]
    x = torch.randn(shape, generator=g, device="cuda") * (torch.rand(c, generator=g, device="cuda") + 0.5)
    x = (x + offset * torch.randn(c, generator=g, device="cuda")).to(DT[dtype])
    gamma = (torch.rand(c, generator=g, device="cuda") + 0.5).to(DT[param])
    beta = (0.3 * torch.randn(c, generator=g, device="cuda")).to(DT[param])
    dy = (0.1 * torch.randn(shape, generator=g, device="cuda")).to(DT[dtype])
    return x, gamma, beta, dy


def away_from_kink(x, gamma, beta, groups):
    """ReLU's derivative jumps at 0: move the few inputs whose z is within the error of one rounding of it."""
    r = reference(x, gamma, beta, groups, "none")["y"][0]
    return torch.where(r.abs() < 1e-3, x.float() + 0.05, x.float()).to(x.dtype)


SHAPES = [   # [batch, ..., channels], groups
    ((1, 1, 1, 8), 1),
    ((1, 1, 1, 4), 4),                # groups of one value: variance 0, rstd = 1/sqrt(eps)
    ((2, 3, 5, 6), 2),
    ((3, 7, 11, 30), 3),
    ((2, 1, 1, 512), 32),
    ((4, 4, 4, 512), 32),
    ((2, 32, 32, 64), 32),
    ((1, 19, 23, 90), 9),
    ((2, 40, 40, 96), 1),             # one group
    ((1, 9, 9, 1030), 2),             # groups wider than a block's columns
    ((1, 100, 130, 16), 4),           # long images
    ((1, 257, 256, 40), 5),
    ((5, 33), 11),                    # no pixel dimensions
    ((130, 2, 2, 24), 8),
    ((1, 128, 128, 256), 1),          # a group far larger than shared memory
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,param", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp16", "fp16")])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_forward_and_backward_match_64_bits(case, dtype, param):
    shape, groups = SHAPES[case]
    for act in ("none", "relu", "silu"):
        x, gamma, beta, dy = inputs(shape, dtype, param, seed=case)
        if act == "relu":
            x = away_from_kink(x, gamma, beta, groups)
        want = reference(x, gamma, beta, groups, act, dy)
        y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, groups, EPS, act)
        for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
            close(got, want[name])
        if act == "relu" and float(want["z_err"]) < 1:
            continue      # an input on the kink after all (groups of one value)
        dx, dgamma, dbeta = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, groups, act)
        for got, name in ((dx, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
            close(got, want[name])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_channel_slices_odd_addresses_and_missing_parameters(dtype):
    wide, _, _, dy = inputs((3, 6, 7, 48), dtype, "fp32", seed=1)
    for lo, hi, groups in ((0, 16, 4), (8, 24, 2), (3, 21, 3), (47, 48, 1)):
        x, d = wide[..., lo:hi], dy[..., lo:hi]
        want = reference(x, None, None, groups, "silu", d)
        y, mean, rstd = hdqt.group_norm_fwd(x, None, None, groups, EPS, "silu")
        assert y.is_contiguous()
        close(y, want["y"])
        dx, dgamma, dbeta = hdqt.group_norm_bwd(d, x, None, None, mean, rstd, groups, "silu")
        assert dgamma is None and dbeta is None
        close(dx, want["dx"])
    x = wide[:, ::2, :, :][:, :, :, 0:16][1:2]      # one row of the batch, rows apart: not evenly spaced
    with pytest.raises(ValueError):
        hdqt.group_norm_fwd(x, None, None, 4)
    x = wide[:, 2:3, ::2, 0:16]                     # one image row, every other pixel: evenly spaced
    close(hdqt.group_norm_fwd(x, None, None, 4)[0], reference(x, None, None, 4, "none")["y"])


@pytest.mark.gpu
def test_large_mean_and_constant_groups():
    x, gamma, beta, dy = inputs((2, 16, 16, 32), "fp32", "fp32", seed=3)
    x = x + 1000.0
    want = reference(x, gamma, beta, 8, "none", dy)
    y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 8, EPS)
    close(y, want["y"])
    # the variance itself must not lose digits to the mean: what is lost is the rounding of the inputs' distance from it
    assert float((rstd.double() / want["rstd"][0] - 1).abs().max()) < 1e-5
    const = torch.full((1, 5, 5, 8), 3.0, device="cuda")
    y, mean, rstd = hdqt.group_norm_fwd(const, gamma[:8], beta[:8], 2, EPS)
    assert torch.equal(y, beta[:8].expand_as(y)) and bool((mean == 3).all())
    assert float((rstd - EPS ** -0.5).abs().max()) < 1e-3


@pytest.mark.gpu
def test_gradient_matches_differences():
    """<grad, v> against (L(+h v) - L(-h v)) / 2h with h = 2^-5 and L formed in 64 bits from the call's outputs: the
    third-derivative term is h^2/6 = 1.6e-4 times O(1), the rounding of L e sqrt(n) |y| / h = 1e-4 of |v||c|."""
    x, gamma, beta, dy = inputs((2, 5, 6, 24), "fp32", "fp32", seed=9)
    g = torch.Generator(device="cuda").manual_seed(1)
    for act in ("none", "silu"):
        y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 4, EPS, act)
        grads = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, 4, act)
        for which, grad in enumerate(grads):
            args = [x, gamma, beta]
            v = torch.randn(args[which].shape, generator=g, device="cuda")
            h, loss = 2.0 ** -5, []
            for sign in (1, -1):
                moved = list(args)
                moved[which] = args[which] + sign * h * v
                loss.append(float((hdqt.group_norm_fwd(*moved, 4, EPS, act)[0].double() * dy.double()).sum()))
            want = (loss[0] - loss[1]) / (2 * h)
            scale = float(dy.norm()) * float(v.norm())
            assert abs(float((grad.double() * v.double()).sum()) - want) <= 1e-3 * scale


@pytest.mark.gpu
def test_non_finite_values_stay_in_their_group():
    x, gamma, beta, dy = inputs((2, 4, 4, 16), "fp32", "fp32", seed=4)
    x[1, 2, 2, 5] = math.nan
    y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 4, EPS, "silu")
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[1, :, :, 4:8] = True
    assert torch.equal(torch.isnan(y), bad)
    x[1, 2, 2, 5] = math.inf
    y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 4, EPS, "relu")
    assert torch.equal(torch.isnan(y), bad)


@pytest.mark.gpu
def test_empty_batches_and_images():
    gamma, beta = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    for shape in ((0, 3, 3, 8), (2, 0, 3, 8)):
        x = torch.empty(shape, device="cuda")
        y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 2)
        assert y.shape == x.shape and mean.shape == (shape[0], 2) and bool(torch.isnan(mean).all())
        dx, dgamma, dbeta = hdqt.group_norm_bwd(x, x, gamma, beta, mean, rstd, 2)
        assert dx.shape == x.shape and not dgamma.any() and not dbeta.any()


@pytest.mark.gpu
def test_parts_of_the_gradient_and_repeatability():
    x, gamma, beta, dy = inputs((3, 9, 9, 32), "bf16", "fp32", seed=5)
    y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 8, EPS, "silu")
    dx, dgamma, dbeta = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, 8, "silu")
    only_dx = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, 8, "silu", want_params=False)
    only_params = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, 8, "silu", want_dx=False)
    assert torch.equal(only_dx[0], dx) and only_dx[1] is None and only_params[0] is None
    assert torch.equal(only_params[1], dgamma) and torch.equal(only_params[2], dbeta)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, 8, "silu")
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dgamma, dbeta)))


def test_refusals():
    with pytest.raises(ValueError):
        hdqt.group_norm_fwd(torch.zeros(2, 3, 3, 8), None, None, 2)            # not on a GPU
    import ctypes as C
    lib = hdqt.lib
    INVALID, UNSUPPORTED, ALIGN, WS = 1, 2, 3, 4

    def desc(**over):
        d = hdqt.GroupNormDesc(2, 9, 16, 4, 144, 16, 144, 16, 0, 0, 0, 1e-5)
        for k, v in over.items():
            setattr(d, k, v)
        return d

    def fwd(d, x=256, y=256, gamma=256, mean=256, ws=256, ws_bytes=1 << 20):
        return lib.hdqt_group_norm_fwd(C.byref(d), x, gamma, 256, y, mean, 256, ws, ws_bytes, None)

    for bad in ({"channels": 0}, {"groups": 0}, {"groups": 3}, {"batch": -1}, {"pixels": -1}, {"dtype": 7},
                {"param_dtype": 1}, {"act": 3}, {"act": -1}, {"eps": -1.0}, {"eps": math.nan}, {"x_pixel_stride": 15},
                {"x_batch_stride": 143}, {"y_pixel_stride": 8}, {"y_batch_stride": 10}):
        assert fwd(desc(**bad)) == INVALID, bad
    assert fwd(desc(channels=1 << 21, groups=1, x_pixel_stride=1 << 21, y_pixel_stride=1 << 21, x_batch_stride=1 << 30,
                    y_batch_stride=1 << 30)) == UNSUPPORTED
    assert fwd(desc(), x=None) == INVALID and fwd(desc(), y=None) == INVALID and fwd(desc(), mean=None) == INVALID
    assert fwd(desc(), x=258) == ALIGN and fwd(desc(), gamma=257) == ALIGN and fwd(desc(), ws=384 + 8) == ALIGN
    assert fwd(desc(), ws_bytes=8) == WS
    assert lib.hdqt_group_norm_bwd(C.byref(desc()), None, 256, 256, 256, 256, 256, 256, 256, 256, 256, 1 << 20, None) == INVALID
    assert lib.hdqt_group_norm_bwd(C.byref(desc()), 256, 256, 256, 256, 256, 256, 256, 258, 256, 256, 1 << 20, None) == ALIGN
    assert lib.hdqt_group_norm_bwd(C.byref(desc()), 256, 256, 256, 256, 256, 256, 256, 256, 256, 256, 8, None) == WS
    assert lib.hdqt_group_norm_workspace_bytes(C.byref(desc(groups=5)), 0) == 0


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """2.3e9 elements: the last image's groups against 64 bits (statistics of a group: 2^20 x 44 values, summed per thread over at
    most a few thousand of them: the bounds of the docstring with room for the longer sums)."""
    b, p, c, groups = 2, 1 << 20, 1100, 25
    x = torch.empty((b, p, c), dtype=torch.bfloat16, device="cuda")
    for i in range(b):
        x[i].normal_(0.5, 1.0)
    y, mean, rstd = hdqt.group_norm_fwd(x, None, None, groups, EPS, "relu")
    dx, _, _ = hdqt.group_norm_bwd(x, x, None, None, mean, rstd, groups, "relu", want_params=False)
    for g in (0, groups - 1):
        xs = x[1, :, g * 44:(g + 1) * 44].double()
        mu, rs = xs.mean(), (xs.var(correction=0) + EPS) ** -0.5
        assert abs(float(mean[1, g]) - float(mu)) < 1e-4 and abs(float(rstd[1, g] / rs) - 1) < 1e-4
        z = (xs - mu) * rs
        got = y[1, :, g * 44:(g + 1) * 44].double()
        assert float((got - z.clamp_min(0)).abs().max()) < 2.0 ** -8 * float(z.max()) + 1e-3
        dz = torch.where(z > 0, xs, 0.0)
        want = rs * (dz - dz.mean() - z * (dz * z).mean())
        far = (dx[1, :, g * 44:(g + 1) * 44].double() - want).abs() > 2.0 ** -8 * want.abs() + 1e-2
        assert float(far.double().mean()) < 1e-4          # (elements on ReLU's kink)
        del xs, z, got, dz, want, far
