"""The step operators through autograd and the training loops: modules and functions of nn.py against torch's own, a model
that runs them together, and the same step replayed from CUDA graphs."""
import math

import pytest
import torch

from paper_2310_03675_b200 import nn as hnn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["nhwc", "nchw"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_group_norm_module_matches_torch_in_64_bits(act, layout):
    torch.manual_seed(0)
    m = hnn.GroupNormAct(24, groups=6, act=act).cuda()
    with torch.no_grad():
        m.weight.uniform_(0.5, 1.5)
        m.bias.normal_(0, 0.3)
    x = torch.randn(3, 24, 5, 7, device="cuda")
    if layout == "nhwc":
        x = x.contiguous(memory_format=torch.channels_last)
    x.requires_grad_(True)
    dy = torch.randn(3, 24, 5, 7, device="cuda")
    y = m(x)
    y.backward(dy)
    xd = x.detach().double().requires_grad_(True)
    w, b = m.weight.detach().double().requires_grad_(True), m.bias.detach().double().requires_grad_(True)
    z = torch.nn.functional.group_norm(xd, 6, w, b, m.eps)
    ref = {"none": z, "relu": torch.relu(z), "silu": torch.nn.functional.silu(z)}[act]
    ref.backward(dy.double())
    # outputs and gradients are sums of at most 140 O(1) terms in fp32 (2^-24 each): well inside 140 * 2^-24 = 8e-6
    for got, want in ((y, ref), (x.grad, xd.grad), (m.weight.grad, w.grad), (m.bias.grad, b.grad)):
        assert float((got.double() - want).detach().abs().max()) < 2e-5 * max(1.0, float(want.detach().abs().max()))


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("bias", [False, True])
def test_linear_cross_entropy_matches_torch_in_64_bits(reduction, bias):
    torch.manual_seed(1)
    for t, d, v in ((60, 40, 30), (600, 72, 700)):
        x = torch.randn(t, d, device="cuda", requires_grad=True)
        w = (torch.randn(d, v, device="cuda") / math.sqrt(d)).requires_grad_(True)
        b = torch.randn(v, device="cuda", requires_grad=True) if bias else None
        labels = torch.randint(0, v, (t,), device="cuda")
        labels[::7] = -100
        up = torch.randn(t, device="cuda") if reduction == "none" else torch.tensor(0.3, device="cuda")
        loss = hnn.linear_cross_entropy(x, w, labels, bias=b, reduction=reduction)
        loss.backward(up, retain_graph=True)
        xd, wd = x.detach().double().requires_grad_(True), w.detach().double().requires_grad_(True)
        bd = b.detach().double().requires_grad_(True) if bias else None
        z = xd @ wd if bd is None else xd @ wd + bd
        ref = torch.nn.functional.cross_entropy(z, labels, reduction=reduction)
        ref.backward(up.double())
        # fp32 sums of up to 700 terms: 700 * 2^-24 = 4e-5 of the terms' size, the results are at least a tenth of it
        pairs = [(loss, ref), (x.grad, xd.grad), (w.grad, wd.grad)] + ([(b.grad, bd.grad)] if bias else [])
        for got, want in pairs:
            assert float((got.double() - want).detach().abs().max()) < 5e-5 * float(want.detach().abs().max())
        loss.backward(up)                      # a second pass through the same graph adds the same gradient
        assert float((x.grad.double() - 2 * xd.grad).abs().max()) < 1e-4 * float(xd.grad.abs().max())


def test_linear_cross_entropy_without_some_gradients():
    torch.manual_seed(2)
    x, w = torch.randn(9, 16, device="cuda"), torch.randn(16, 20, device="cuda")
    labels = torch.randint(0, 20, (9,), device="cuda")
    plain = hnn.linear_cross_entropy(x, w, labels)
    assert not plain.requires_grad
    wp = w.clone().requires_grad_(True)
    loss = hnn.linear_cross_entropy(x, wp, labels)
    loss.backward()
    assert loss.item() == plain.item() and wp.grad is not None
    xp = x.clone().requires_grad_(True)
    hnn.linear_cross_entropy(xp, w, labels).backward()
    assert xp.grad is not None


@pytest.mark.parametrize("norm_type", [2.0, math.inf])
def test_clip_grad_norm_matches_torch(norm_type):
    torch.manual_seed(3)
    params = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((3, 5), (7,), (4, 3, 3, 3))]
    params.append(torch.nn.Parameter(torch.randn(2, device="cuda")))            # has no gradient
    for p in params[:3]:
        p.grad = torch.randn_like(p)
    params[2].grad = params[2].grad.contiguous(memory_format=torch.channels_last)   # dense, permuted
    ref = [torch.nn.Parameter(p.detach().clone()) for p in params]
    for p, q in zip(params[:3], ref):
        q.grad = p.grad.clone()
    want = torch.nn.utils.clip_grad_norm_(ref, 0.5, norm_type)
    got = hnn.clip_grad_norm_(params, 0.5, norm_type)
    assert abs(float(got) - float(want)) <= 1e-6 * float(want)
    for p, q in zip(params[:3], ref):
        assert float((p.grad - q.grad).abs().max()) <= 1e-6 * float(q.grad.abs().max())
    params[0].grad = torch.randn(10, 10, device="cuda")[::2, ::2].t()[:3, :5]
    with pytest.raises(ValueError):
        hnn.clip_grad_norm_([params[0]], 1.0)


def test_network_gradients_through_the_operators_match_torch(monkeypatch):
    """The network with its matrix products in fp32: loss and all gradients through the operators against the same network on
    torch's group norm and cross entropy in 64 bits (sums of 1e4..1e5 terms through 20 layers in fp32: 1e-3 of a tensor's norm)."""
    monkeypatch.setattr(torch.backends.cudnn, "allow_tf32", False)
    torch.manual_seed(4)
    model = hnn.ResNet18Width(12, quantized=False, widths=(32, 32, 64, 64), norm="group").cuda()
    y = torch.randint(0, 12, (16,), device="cuda")
    x = hnn.synthetic_images(y, hnn.class_patterns(12, 4, "cuda"), seed=4)
    loss = model.loss(x, y)
    loss.backward()
    got = {n: p.grad.double() for n, p in model.named_parameters()}

    def forward(self, v):
        z = torch.nn.functional.group_norm(v, self.groups, self.weight, self.bias, self.eps)
        return torch.relu(z) if self.act == "relu" else z

    monkeypatch.setattr(hnn.GroupNormAct, "forward", forward)
    model.double()
    model.zero_grad(set_to_none=True)
    ref = torch.nn.functional.cross_entropy(model(x.double()), y)
    ref.backward()
    assert abs(loss.item() - ref.item()) < 1e-5 * abs(ref.item())
    for n, p in model.named_parameters():
        assert float((got[n] - p.grad).norm()) < 1e-3 * float(p.grad.norm()), n


@pytest.mark.parametrize("graphed", [False, True])
def test_quantized_step_with_the_operators_lowers_the_loss(graphed):
    torch.manual_seed(5)
    model = hnn.ResNet18Width(12, widths=(32, 32, 64, 64), norm="group").cuda()
    y = torch.randint(0, 12, (64,), device="cuda")
    x = hnn.synthetic_images(y, hnn.class_patterns(12, 5, "cuda"), seed=5)
    lr, clip = 0.05, 1.0
    opt = torch.optim.SGD(model.parameters(), lr=lr)
    stepper = hnn.GraphedTrainStep(model, opt, x, y, loss=model.loss, clip_norm=clip) if graphed else None
    losses = []
    for step in range(40):
        before = [p.detach().clone() for p in model.parameters()]
        loss = stepper(x, y) if graphed else hnn.cnn_train_step(model, opt, x, y, step, fused_loss=True, clip_norm=clip)
        losses.append(loss.item())
        moved = math.sqrt(sum(float((p.detach() - q).double().square().sum()) for p, q in zip(model.parameters(), before)))
        assert moved <= lr * clip * 1.001          # the update is lr times the clipped gradient
    assert all(math.isfinite(v) for v in losses)
    assert sum(losses[-10:]) < sum(losses[:10])


def test_class_incremental_run_with_the_step_operators():
    for graphed in (False, True):
        out = hnn.class_incremental_run(True, "cuda", tasks=2, classes_per_task=3, steps_per_task=6, batch=32, memory=30,
                                        test_per_class=2, norm="group", fused_loss=True, clip_norm=1.0, graphed=graphed)
        assert len(out["accuracy_after_task"]) == 2 and all(0.0 <= a <= 1.0 for a in out["accuracy_after_task"])
