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
