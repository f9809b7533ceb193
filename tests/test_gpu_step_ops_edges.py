"""Edges of the step operators on the GPU: bf16 through autograd, tensors of another device than the current one, extreme values,
and the kernel variants that only particular sizes reach."""
import math

import pytest
import torch

from paper_2310_03675_b200 import hdqt
from paper_2310_03675_b200 import nn as hnn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,features,classes", [(60, 40, 30), (600, 72, 700)])
def test_bf16_gradients_through_autograd(tokens, features, classes):
    """dX = dz W and dW = dz^T X.  Error of an element, in units of S = sum |dz| |w|: dz rounded to bf16 2^-8, its code 2^-12, the
    fp32 sums of at most 700 terms 700 * 2^-24 < 2^-14, the result 2^-8 of itself <= 2^-8 S, and where an unstated factor arrives
    another 2^-8 S."""
    torch.manual_seed(6)
    x = torch.randn(tokens, features, device="cuda").bfloat16().requires_grad_(True)
    w = (torch.randn(features, classes, device="cuda") / math.sqrt(features)).bfloat16().requires_grad_(True)
    labels = torch.randint(0, classes, (tokens,), device="cuda")
    labels[::7] = -100
    kept = int((labels != -100).sum())
    p = torch.softmax(x.detach().double() @ w.detach().double(), 1)
    hot = torch.zeros_like(p)
    hot[torch.arange(tokens, device="cuda"), labels.clamp_min(0)] = 1.0
    dz = (p - hot) * (0.3 / kept) * (labels != -100)[:, None]
    xd, wd = x.detach().double(), w.detach().double()
    want = (dz @ wd.t(), xd.t() @ dz)
    size = (dz.abs() @ wd.abs().t(), xd.abs().t() @ dz.abs())

    def check(roundings):
        for got, value, s in zip((x.grad, w.grad), want, size):
            assert bool(((got.double() - value).abs() <= ((1 + roundings) * 2.0 ** -8 + 2.0 ** -11) * s).all())

    loss = hnn.linear_cross_entropy(x, w, labels)
    loss.backward(torch.tensor(0.3, device="cuda"), retain_graph=True)       # a factor that was not known: rounded twice
    check(2)
    x.grad = w.grad = None
    loss.backward(torch.tensor(0.3, device="cuda"))                          # the retained graph
    check(1)
    x.grad = w.grad = None
    scaled = hnn.linear_cross_entropy(x, w, labels, scale=0.3)
    assert abs(scaled.item() - 0.3 * loss.item()) <= 1e-6 * loss.item()
    scaled.backward()
    check(1)
    g = torch.tensor(0.3, device="cuda")
    _, _, dx, dw = hdqt.linear_xent_train(x.detach(), w.detach(), labels, g)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw)               # the bits of the call that rounds once


def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    """With the current device reported as another one every call enters the tensors' own, and gives the same bits."""
    torch.manual_seed(7)
    x, w = torch.randn(70, 40, device="cuda"), torch.randn(40, 50, device="cuda")
    labels = torch.randint(0, 50, (70,), device="cuda")
    img, dy = torch.randn(2, 3, 3, 16, device="cuda"), torch.randn(2, 3, 3, 16, device="cuda")

    def everything():
        y, mean, rstd = hdqt.group_norm_fwd(img, None, None, 4)
        dx = hdqt.group_norm_bwd(dy, img, None, None, mean, rstd, 4)[0]
        loss, lse = hdqt.linear_xent_fwd(x, w, labels)
        grads = hdqt.linear_xent_bwd(x, w, labels, lse) + hdqt.linear_xent_train(x, w, labels)
        clipped = [x.clone()]
        norm = hdqt.clip_grad_norm(clipped, 1.0)
        hdqt.scale_tensors(clipped, norm)
        return y, mean, rstd, dx, loss, lse, *grads, norm, clipped[0], hdqt.grad_norm([x]), hdqt.gemm_fwd(x, w)[0]

    want = everything()
    entered = []
    real = torch.cuda.device

    class Guard(real):
        def __init__(self, index):
            entered.append(index)
            super().__init__(index)

    monkeypatch.setattr(hdqt, "_raw_device", lambda: 7)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    got = everything()
    assert len(entered) == 9 and set(entered) == {0}
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError):
        hdqt.calibrate_acc_shift(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 32, dtype=torch.int8))


def test_fp32_values_above_the_largest_bf16_value():
    """fp32 operands travel as three bf16 planes; a mask of the lowest fp32 value rounds to -infinity in the first of them.  Classes
    that no token may take leave loss and gradients those of the other classes; 300 x 32 x 400, O(1) logits.  Tolerances: 32 products
    of 24 bits, sums of at most 400 terms with 2^-23 dropped at each of 400/16 additions: 1e-5 of the terms' size, which is
    below 40 for a gradient."""
    g = torch.Generator(device="cuda").manual_seed(8)
    low = torch.finfo(torch.float32).min
    x = torch.randn(300, 32, generator=g, device="cuda")
    w = torch.randn(400, 32, generator=g, device="cuda") * 0.25
    x[:, 0] = 1.0
    w[:, 0] = 0.0
    w[100:, 0] = low
    labels = torch.randint(0, 100, (300,), generator=g, device="cuda")
    rows = torch.rand(300, generator=g, device="cuda")
    xd, wd = x[:, 1:].double(), w[:100, 1:].double()
    z = xd @ wd.t()
    lse = torch.logsumexp(z, 1)
    dz = torch.softmax(z, 1)
    dz[torch.arange(300), labels] -= 1.0
    dz *= rows.double()[:, None]
    for piece in (0, 1 << 28):
        how = {"reduction": "none", "w_is_cd": True, "piece_bytes": piece}
        loss, got_lse, dx, dw = hdqt.linear_xent_train(x, w, labels, rows, **how)
        dx2, dw2 = hdqt.linear_xent_bwd(x, w, labels, got_lse, rows, **how)
        assert float((got_lse.double() - lse).abs().max()) < 1e-5
        assert float((loss.double() - (lse - z.gather(1, labels[:, None])[:, 0])).abs().max()) < 1e-5
        for a, b in ((dx, dw), (dx2, dw2)):
            assert not b[100:].any()
            assert float((a[:, 1:].double() - dz @ wd).abs().max()) < 4e-4
            assert float((b[:100, 1:].double() - dz.t() @ xd).abs().max()) < 4e-4
    x[5, 3], w[7, 3] = 3.4e38, 0.0                       # a large activation against a class that does not look at it
    z = x.double()[5] @ w.double()[7]
    _, got_lse, _, _ = hdqt.linear_xent_train(x, w[7:8].contiguous(), torch.zeros_like(labels), rows, **how)
    assert abs(float(got_lse[5].double() - z)) < 1e-5


@pytest.mark.parametrize("shape", [(2, 3, 0, 8), (2, 0, 0, 8), (0, 3, 0, 8), (3, 0, 8)])
def test_group_norm_of_images_without_pixels(shape):
    gamma, beta = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    x = torch.empty(shape, device="cuda")
    y, mean, rstd = hdqt.group_norm_fwd(x, gamma, beta, 2)
    assert y.shape == x.shape and mean.shape == (shape[0], 2) and bool(torch.isnan(mean).all())
    dx, dgamma, dbeta = hdqt.group_norm_bwd(x, x, gamma, beta, mean, rstd, 2)
    assert dx.shape == x.shape and not dgamma.any() and not dbeta.any()


def rounding_ratio(got, want):
    """Error of a bf16 result against 64 bits, over what rounding the exact result leaves."""
    want = want.double()
    return float((got.double() - want).norm() / (want.bfloat16().double() - want).norm())


def weighted_gradients(tokens, features, classes, weights, w_is_cd, seed):
    """Error ratios of dX and dW, backward and one-call form, bf16 with a weight per row.  Beyond the final rounding there is dz's:
    at the label p - 1 with p of 1 / classes, a bf16 number to that fraction of an ulp, elsewhere numbers of size p whose roundings
    add up to 2^-8 / sqrt(classes) of the row.  For 3000 classes and more both together are below a tenth of the final
    rounding's 2^-8 / sqrt(3) (1 / 2) at the worst, so the ratio is at most 1.1 if the weights themselves are not rounded."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(tokens, features, generator=g, device="cuda").bfloat16()
    w = (torch.randn(classes, features, generator=g, device="cuda") / math.sqrt(features)).bfloat16()
    labels = torch.randint(0, classes, (tokens,), generator=g, device="cuda")
    dz = torch.softmax(x.double() @ w.double().t(), 1)
    dz[torch.arange(tokens, device="cuda"), labels] -= 1.0
    dz *= weights.double()[:, None]
    ww = w if w_is_cd else w.t().contiguous()
    how = {"reduction": "none", "w_is_cd": w_is_cd}
    loss, lse = hdqt.linear_xent_fwd(x, ww, labels, **how)
    pairs = (hdqt.linear_xent_bwd(x, ww, labels, lse, weights, **how), hdqt.linear_xent_train(x, ww, labels, weights, **how)[2:])
    return [r for dx, dw in pairs
            for r in (rounding_ratio(dx, dz @ w.double()), rounding_ratio(dw if w_is_cd else dw.t(), dz.t() @ x.double()))]


@pytest.mark.parametrize("w_is_cd", [False, True])
@pytest.mark.parametrize("tokens,classes", [(600, 3000), (2000, 3001)])
def test_equal_row_weights_lose_no_bits(tokens, classes, w_is_cd):
    """What `reduction="none"` and a mean over its losses arrive as.  1 + 2^-8 - 2^-11 lies almost half way between two bf16 numbers."""
    for value in (1 + 2.0 ** -8 - 2.0 ** -11, -(1 + 2.0 ** -8 - 2.0 ** -11) / tokens):
        weights = torch.full((tokens,), value, device="cuda")
        for ratio in weighted_gradients(tokens, 128, classes, weights, w_is_cd, seed=31):
            assert ratio <= 1.1


def test_row_weights_that_are_zero_or_not_finite():
    g = torch.Generator(device="cuda").manual_seed(32)
    x = torch.randn(600, 64, generator=g, device="cuda").bfloat16()
    w = torch.randn(3000, 64, generator=g, device="cuda").bfloat16()
    labels = torch.randint(0, 3000, (600,), generator=g, device="cuda")
    labels[10] = -100
    how = {"reduction": "none", "w_is_cd": True}
    lse = hdqt.linear_xent_fwd(x, w, labels, **how)[1]
    for call in (lambda a: hdqt.linear_xent_bwd(x, w, labels, lse, a, **how), lambda a: hdqt.linear_xent_train(x, w, labels, a, **how)[2:]):
        dx, dw = call(torch.zeros(600, device="cuda"))
        assert not dx.any() and not dw.any()
        weights = torch.full((600,), 1e-38, device="cuda")          # the smallest normal numbers
        dx, dw = call(weights)
        one, _ = call(torch.ones(600, device="cuda"))
        assert float((dx.double() * 1e38 - one.double()).norm() / one.double().norm()) < 2.0 ** -6
        for bad in (math.inf, math.nan):
            weights = torch.ones(600, device="cuda")
            weights[7] = weights[10] = bad                           # (row 10 is ignored: its weight is not looked at)
            dx, dw = call(weights)
            finite = torch.isfinite(dx).all(1)
            assert not bool(finite[7]) and bool(finite[:7].all()) and bool(finite[8:].all())
            assert torch.equal(dx[finite], one[finite]) and not dx[10].any()


@pytest.mark.parametrize("w_is_cd", [False, True])
@pytest.mark.parametrize("tokens,classes", [(9, 9000), (28, 5001), (130, 3000), (256, 3001)])
def test_row_weights_of_a_few_tokens_lose_no_bits(tokens, classes, w_is_cd):
    """Few tokens do not average what rounding each one's weight leaves; all but one lie almost half way between bf16 numbers here."""
    weights = torch.full((tokens,), 0.5 * (1 + 2.0 ** -8 - 2.0 ** -11), device="cuda")
    weights[0] = 1.0
    rand = torch.rand(tokens, generator=torch.Generator(device="cuda").manual_seed(33), device="cuda") - 0.5
    for g in (weights, -3.0 * weights, rand):
        for ratio in weighted_gradients(tokens, 256, classes, g, w_is_cd, seed=34):
            assert ratio <= 1.1


@pytest.mark.parametrize("w_is_cd", [False, True])
def test_row_weights_of_a_few_tokens_in_pieces_and_at_odd_sizes(w_is_cd):
    """Pieces of tokens (one-call form) and of classes (backward), rows that must be copied, ignored rows, non-finite weights of them."""
    import test_gpu_xent as xe
    for t, d, v in ((200, 100, 2003), (256, 67, 1025), (40, 1030, 3000), (257, 64, 20011)):
        x, w, labels, weights = xe.data(t, d, v, "bf16", seed=t)
        ww = w if w_is_cd else w.t().contiguous()
        want = xe.reference(x, w, labels, weights, torch.bfloat16)
        weights[labels == -100] = math.nan                          # not looked at
        how = {"reduction": "none", "w_is_cd": w_is_cd}
        lse = hdqt.linear_xent_fwd(x, ww, labels, **how)[1]
        for piece in (0, 1, 1 << 20):
            dx, dw = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, piece_bytes=piece, **how)
            dx2, dw2 = hdqt.linear_xent_train(x, ww, labels, weights, piece_bytes=piece, **how)[2:]
            only_dx = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, piece_bytes=piece, want_dw=False, **how)[0]
            only_dw = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, piece_bytes=piece, want_dx=False, **how)[1]
            for got, name in ((dx, "dx"), (dx2, "dx"), (only_dx, "dx"), (dw, "dw"), (dw2, "dw"), (only_dw, "dw")):
                xe.close(got if name == "dx" or w_is_cd else got.t(), want[name], name)
