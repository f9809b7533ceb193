"""Kernel variants of the step operators that only particular sizes reach, against 64-bit arithmetic.  Formulas, inputs and bounds
are those of the operators' own tests; every comparison here fails on a NaN."""
import math

import pytest
import torch

import test_gpu_groupnorm as gn
import test_gpu_xent as xe
from paper_2310_03675_b200 import hdqt


def within(got, want, name):
    """|got - value| <= err + one rounding to got's type, NaN nowhere."""
    value, err = want
    tiny = 2.0 ** -25 if got.dtype == torch.float16 else 1e-37
    ok = (got.double() - value).abs() <= err + gn.UNIT[got.dtype] * (value.abs() + err) + tiny
    assert bool(ok.all()), (name, int((~ok).sum()))


def test_the_comparison_fails_on_nan():
    value = torch.tensor([1.0, 2.0], dtype=torch.float64)
    err = torch.full_like(value, 1e-3)
    within(torch.tensor([1.0, 2.0]), (value, err), "equal")
    for bad in (math.nan, 2.1, math.inf):
        with pytest.raises(AssertionError):
            within(torch.tensor([1.0, bad]), (value, err), "bad")


def check_group_norm(shape, groups, dtype, param, act, seed):
    x, gamma, beta, dy = gn.inputs(shape, dtype, param, seed=seed)
    if act == "relu":
        x = gn.away_from_kink(x, gamma, beta, groups)
    want = gn.reference(x, gamma, beta, groups, act, dy)
    y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, groups, gn.EPS, act)
    for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
        within(got, want[name], name)
    dx, dgamma, dbeta = hdqt.group_norm_bwd(dy, x, gamma, beta, mean, rstd, groups, act)
    kink = act == "relu" and not float(want["z_err"]) >= 1      # (groups of one value)
    for got, name in ((dx, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
        if kink:
            assert bool(torch.isfinite(got).all()), name
        else:
            within(got, want[name], name)


TYPES = [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp16", "fp16")]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,param", TYPES)
@pytest.mark.parametrize("case", range(len(gn.SHAPES)))
def test_group_norm_is_within_its_bounds_and_nowhere_nan(case, dtype, param):
    for act in ("none", "relu", "silu"):
        check_group_norm(*gn.SHAPES[case], dtype, param, act, seed=case)


# groups wider than a block's 256 columns, by the channels of an access (8, 4, 2, 1 of 16 bits; 4, 2, 1 of 32), images of one and of
# several chunks of pixels
WIDE_GROUPS = [
    ((2, 5, 7, 4160), 2),
    ((1, 19, 29, 4160), 2),
    ((3, 1, 1, 2056), 1),
    ((1, 31, 33, 1028), 1),
    ((2, 17, 16, 1030), 1),
    ((2, 6, 7, 771), 3),
    ((1, 40, 26, 257), 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,param", TYPES)
@pytest.mark.parametrize("case", range(len(WIDE_GROUPS)))
def test_group_norm_of_wide_groups(case, dtype, param):
    for act in ("none", "relu", "silu"):
        check_group_norm(*WIDE_GROUPS[case], dtype, param, act, seed=100 + case)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_channel_slices_of_wide_groups(dtype):
    """Bases and strides that allow 8, 4, 2 and 1 elements at a time."""
    wide, _, _, dy = gn.inputs((2, 9, 11, 4200), dtype, "fp32", seed=120)
    for off in (0, 4, 2, 1):
        x, d = wide[..., off:off + 4160], dy[..., off:off + 4160]
        want = gn.reference(x, None, None, 2, "silu", d)
        y, mean, rstd = hdqt.group_norm_fwd(x, None, None, 2, gn.EPS, "silu")
        dx, _, _ = hdqt.group_norm_bwd(d, x, None, None, mean, rstd, 2, "silu")
        for got, name in ((y, "y"), (mean, "mean"), (rstd, "rstd"), (dx, "dx")):
            within(got, want[name], name)


@pytest.mark.gpu
def test_large_tensors_leave_no_element_unwritten():
    """2.3e9 elements: every output is finite (the values of its groups are compared in the operator's own test)."""
    b, p, c, groups = 2, 1 << 20, 1100, 25
    x = torch.empty((b, p, c), dtype=torch.bfloat16, device="cuda")
    for i in range(b):
        x[i].normal_(0.5, 1.0)
    y, mean, rstd = hdqt.group_norm_fwd(x, None, None, groups, gn.EPS, "relu")
    dx, _, _ = hdqt.group_norm_bwd(x, x, None, None, mean, rstd, groups, "relu", want_params=False)
    assert bool(torch.isfinite(mean).all()) and bool(torch.isfinite(rstd).all())
    for t in (y, dx):
        for i in range(b):
            for part in t[i].chunk(8):
                assert bool(torch.isfinite(part).all())


# tokens, features, classes
STREAMED = [(9, 264, 6001), (16, 100, 7001), (13, 520, 3000), (12, 1030, 4096), (3, 264, 6001), (2, 1030, 4099)]
SPLIT_LOGITS = [(2500, 4096, 70), (200, 4096, 3000), (700, 4096, 1100), (130, 6200, 900)]


def check_cross_entropy(t, d, v, dtype, w_is_cd, seed):
    x, w, labels, weights = xe.data(t, d, v, dtype, seed=seed)
    ww = w if w_is_cd else w.t().contiguous()
    want = xe.reference(x, w, labels, weights, xe.DT[dtype])
    status = hdqt.new_status("cuda")
    how = {"reduction": "none", "w_is_cd": w_is_cd, "dev_status": status}
    flip = (lambda m: m) if w_is_cd else (lambda m: m.t())
    loss, lse = hdqt.linear_xent_fwd(x, ww, labels, **how)
    dx, dw = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, **how)
    loss2, lse2, dx2, dw2 = hdqt.linear_xent_train(x, ww, labels, weights, **how)
    only_dx = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, want_dw=False, **how)[0]
    only_dw = hdqt.linear_xent_train(x, ww, labels, weights, want_dx=False, **how)[3]
    for got, name in ((loss, "loss"), (lse, "lse"), (dx, "dx"), (flip(dw), "dw"), (loss2, "loss"), (lse2, "lse"), (dx2, "dx"),
                      (flip(dw2), "dw"), (only_dx, "dx"), (flip(only_dw), "dw")):
        xe.close(got, want[name], name)
    hdqt.check_device_status(status)


@pytest.mark.gpu
@pytest.mark.parametrize("w_is_cd", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(STREAMED)))
def test_cross_entropy_gradients_of_a_few_tokens(case, dtype, w_is_cd):
    check_cross_entropy(*STREAMED[case], dtype, w_is_cd, seed=200 + case)


@pytest.mark.gpu
@pytest.mark.parametrize("w_is_cd", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(SPLIT_LOGITS)))
def test_cross_entropy_with_split_logits(case, dtype, w_is_cd):
    """Long contractions and few output blocks: rows of a warp, of 256 and of 1024 threads."""
    check_cross_entropy(*SPLIT_LOGITS[case], dtype, w_is_cd, seed=220 + case)
