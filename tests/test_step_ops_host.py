"""Host side of the step operators (autograd functions, argument checks) on the CPU: the library calls are replaced by plain torch
where a result is needed, and by a recorder where only the arguments matter.  Nothing is launched."""
import pytest
import torch

from paper_2310_03675_b200 import hdqt
from paper_2310_03675_b200 import nn as hnn


@pytest.fixture
def plain_calls(monkeypatch):
    """group_norm_* (no activation) and linear_xent_* (mean, sum) as torch formulas on CPU tensors; a list of the loss's calls."""
    calls = []

    def gn_fwd(x, gamma, beta, groups, eps, act):
        with torch.no_grad():
            v = x.flatten(1, -2).unflatten(2, (groups, -1))
            mean, var = v.mean((1, 3)), v.var((1, 3), correction=0)
            rstd = (var + eps) ** -0.5
            xh = (v - mean[:, None, :, None]) * rstd[:, None, :, None]
            return (xh.flatten(2) * gamma + beta).view(x.shape), mean, rstd

    def gn_bwd(dy, x, gamma, beta, mean, rstd, groups, act, want_dx=True, want_params=True):
        with torch.enable_grad():
            xs = [t.detach().requires_grad_(True) for t in (x, gamma, beta)]
            v = xs[0].flatten(1, -2).unflatten(2, (groups, -1))
            xh = (v - v.mean((1, 3), keepdim=True)) * (v.var((1, 3), correction=0, keepdim=True) + 1e-5) ** -0.5
            y = (xh.flatten(2) * xs[1] + xs[2]).view(x.shape)
            return torch.autograd.grad(y, xs, dy.detach())

    def loss_and_grads(x, w, labels, g, ignore_index, reduction, w_is_cd):
        with torch.enable_grad():
            xs = [t.detach().float().requires_grad_(True) for t in (x, w)]
            z = xs[0] @ (xs[1].t() if w_is_cd else xs[1])
            loss = torch.nn.functional.cross_entropy(z, labels, ignore_index=ignore_index, reduction=reduction)
            dx, dw = torch.autograd.grad(loss, xs, torch.ones_like(loss) if g is None else g.detach())
        return loss.detach(), dx.to(x.dtype), dw.to(w.dtype), torch.logsumexp(z.detach(), 1)

    def xent_fwd(x, w, labels, ignore_index=-100, reduction="mean", w_is_cd=False):
        calls.append(("fwd", None))
        z = x.detach().float() @ (w.detach().float().t() if w_is_cd else w.detach().float())
        return torch.nn.functional.cross_entropy(z, labels, ignore_index=ignore_index, reduction=reduction), torch.logsumexp(z, 1)

    def xent_train(x, w, labels, g=None, ignore_index=-100, reduction="mean", w_is_cd=False, want_dx=True, want_dw=True):
        calls.append(("train", None if g is None else float(g)))
        loss, dx, dw, lse = loss_and_grads(x, w, labels, g, ignore_index, reduction, w_is_cd)
        return loss, lse, dx if want_dx else None, dw if want_dw else None

    def xent_bwd(x, w, labels, lse, g=None, ignore_index=-100, reduction="mean", w_is_cd=False, want_dx=True, want_dw=True):
        calls.append(("bwd", g if g is None or g.dim() else float(g)))
        _, dx, dw, _ = loss_and_grads(x, w, labels, g, ignore_index, reduction, w_is_cd)
        return dx if want_dx else None, dw if want_dw else None

    def scale(tensors, factor, out=None):
        calls.append(("scale", float(factor)))
        for t in tensors:
            t.copy_((t.float() * factor).to(t.dtype))

    for name, f in (("group_norm_fwd", gn_fwd), ("group_norm_bwd", gn_bwd), ("linear_xent_fwd", xent_fwd),
                    ("linear_xent_train", xent_train), ("linear_xent_bwd", xent_bwd), ("scale_tensors", scale)):
        monkeypatch.setattr(hdqt, name, f)
    return calls


def test_group_norm_refuses_second_derivatives(plain_calls):
    torch.manual_seed(0)
    m = hnn.GroupNormAct(8, groups=2)
    x = torch.randn(2, 8, 3, 3, requires_grad=True)
    y = m(x)
    loss = y.square().mean() + y.pow(3).mean()
    (dx,) = torch.autograd.grad(loss, x, create_graph=True)
    ref = torch.nn.functional.group_norm(x, 2, m.weight, m.bias)
    (want,) = torch.autograd.grad(ref.square().mean() + ref.pow(3).mean(), x)
    assert torch.allclose(dx, want, atol=1e-5)                   # the gradient itself is there
    with pytest.raises(RuntimeError, match="second"):
        (loss + dx.square().sum()).backward()
    m(x).sum().backward()                                        # first derivatives as before
    assert x.grad is not None and m.weight.grad is not None


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_cross_entropy_refuses_second_derivatives(plain_calls, reduction):
    torch.manual_seed(1)
    x, w = torch.randn(6, 4, requires_grad=True), torch.randn(4, 5, requires_grad=True)
    labels = torch.randint(0, 5, (6,))
    loss = hnn.linear_cross_entropy(x, w, labels, reduction=reduction).sum()
    dx, dw = torch.autograd.grad(loss, (x, w), create_graph=True)
    want = torch.autograd.grad(torch.nn.functional.cross_entropy(x @ w, labels, reduction=reduction).sum(), (x, w))
    assert torch.allclose(dx, want[0], atol=1e-6) and torch.allclose(dw, want[1], atol=1e-6)
    for d in (dx, dw):
        with pytest.raises(RuntimeError, match="second"):
            (loss + d.square().sum()).backward(retain_graph=True)
    for t in (x, w):                                             # an input that needs no gradient does not lose the refusal
        other = w if t is x else x
        out = hnn.linear_cross_entropy(*((t, other.detach()) if t is x else (other.detach(), t)), labels, reduction=reduction)
        (d,) = torch.autograd.grad(out.sum(), t, create_graph=True)
        with pytest.raises(RuntimeError, match="second"):
            d.square().sum().backward()


@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_a_known_factor_of_the_loss_is_rounded_with_the_gradients(plain_calls, scale):
    """bf16 gradients are rounded once where the factor is stated: it goes into the call that forms them, and what arrives in the
    backward pass is 1."""
    torch.manual_seed(2)
    x = torch.randn(12, 6).bfloat16().requires_grad_(True)
    w = torch.randn(6, 9).bfloat16().requires_grad_(True)
    labels = torch.randint(0, 9, (12,))
    loss = hnn.linear_cross_entropy(x, w, labels, scale=scale)
    loss.backward(retain_graph=True)
    assert plain_calls == [("train", None if scale == 1.0 else pytest.approx(scale)), ("scale", 1.0)]
    xd, wd = x.detach().double().requires_grad_(True), w.detach().double().requires_grad_(True)
    ref = torch.nn.functional.cross_entropy(xd @ wd, labels) * scale
    ref.backward()
    assert abs(loss.item() - ref.item()) < 1e-6
    first = x.grad.clone(), w.grad.clone()
    for got, want in zip(first, (xd.grad, wd.grad)):
        assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all())       # one rounding (fp32 stand-in)
    loss.backward()                                              # the retained graph: formed again, with the same factor
    assert plain_calls[-1] == ("bwd", pytest.approx(scale))
    for got, want in zip((x.grad, w.grad), first):
        assert torch.equal(got, want * 2)
    per_token = hnn.linear_cross_entropy(x.detach().float(), w.detach().float().requires_grad_(True), labels, reduction="sum", scale=0.5)
    assert per_token.item() == pytest.approx(12 * 0.5 * ref.item() / scale, rel=1e-5)


def test_calls_run_on_the_tensors_device(monkeypatch):
    """A C entry launches on the current device and on the stream it is given: both have to be those of the tensors."""
    log = []

    class Tensor:
        def __init__(self, index):
            self.index = index

        def get_device(self):
            return self.index

    class Guard:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            log.append(("enter", self.index))

        def __exit__(self, *_):
            log.append(("exit", self.index))

    class Lib:
        @staticmethod
        def hdqt_grad_norm(*args):
            log.append(args)
            return 0 if args[0] else 1

        @staticmethod
        def hdqt_status_string(_):
            return b"invalid"

    monkeypatch.setattr(hdqt, "lib", Lib)
    monkeypatch.setattr(hdqt, "_raw_device", lambda: 1)
    monkeypatch.setattr(hdqt, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    hdqt._call("hdqt_grad_norm", Tensor(1), 7)
    assert log == [(7, 1001)]
    log.clear()
    hdqt._call("hdqt_grad_norm", Tensor(0), 7)
    assert log == [("enter", 0), (7, 1000), ("exit", 0)]
    with pytest.raises(hdqt.HdqtError, match="hdqt_grad_norm"):
        hdqt._call("hdqt_grad_norm", Tensor(1), 0)


def test_no_call_takes_the_current_device_for_the_tensors():
    """Every launching C entry goes through hdqt._call; only the rate measurement, which has no tensors, names the stream itself."""
    import inspect
    direct = [line for line in inspect.getsource(hdqt).splitlines() if "_stream()" in line and "def " not in line]
    assert len(direct) == 1 and "hdqt_selftest_mma_rate" in direct[0]


def test_statistics_and_status_words_of_another_device_are_refused(monkeypatch):
    """Their addresses would be read and written by a kernel that cannot reach them."""
    launched = []
    monkeypatch.setattr(hdqt, "_call", lambda name, *args: launched.append(name))
    d = hdqt.GroupNormDesc(2, 9, 16, 4, 144, 16, 144, 16, 0, 0, 0, 1e-5)
    monkeypatch.setattr(hdqt, "_group_norm_plan", lambda *args: (d, (256, 256)))
    x, stat, far = torch.zeros(2, 3, 3, 16), torch.zeros(2, 4), torch.zeros(2, 4, device="meta")
    for mean, rstd in ((far, stat), (stat, far)):
        with pytest.raises(ValueError):
            hdqt.group_norm_bwd(x, x, None, None, mean, rstd, 4)
    hdqt.group_norm_bwd(x, x, None, None, stat, stat, 4)
    assert launched == ["hdqt_group_norm_bwd"]

    launched.clear()
    xd = hdqt.XentDesc(10, 16, 40, 16, 40, 16, 40, -100, 0, 0, 0, 1, 0)
    X, W, labels, lse = torch.zeros(10, 16), torch.zeros(16, 40), torch.zeros(10, dtype=torch.int64), torch.zeros(10)
    monkeypatch.setattr(hdqt, "_xent_call", lambda *args: (X, W, labels, xd, torch.zeros(256, dtype=torch.uint8), 256))
    for status in (torch.zeros(1, dtype=torch.int32, device="meta"), torch.zeros(1), torch.zeros(0, dtype=torch.int32)):
        for call in (lambda: hdqt.linear_xent_fwd(X, W, labels, dev_status=status),
                     lambda: hdqt.linear_xent_bwd(X, W, labels, lse, dev_status=status),
                     lambda: hdqt.linear_xent_train(X, W, labels, dev_status=status)):
            with pytest.raises(ValueError):
                call()
    hdqt.linear_xent_fwd(X, W, labels, dev_status=torch.zeros(1, dtype=torch.int32))
    assert launched == ["hdqt_linear_xent_fwd"]


def test_overlapping_tensors_are_refused_where_they_are_written():
    """Two blocks would read and write the same elements in no fixed order.  Addresses only: the refusal precedes any launch."""
    import ctypes as C
    lib, INVALID = hdqt.lib, 1

    def calls(*entries):
        flat = [v for e in entries for v in e]
        table = (C.c_int64 * len(flat))(*flat)
        return (lib.hdqt_clip_grad_norm(C.addressof(table), len(entries), 2, 1.0, 256, 256, 1 << 20, None),
                lib.hdqt_scale_tensors(C.addressof(table), len(entries), 256, None))

    F32, BF16, A = 0, 1, 1 << 20
    refused = [
        [(A, A, 8, F32), (A, A, 8, F32)],                              # the same tensor twice, in place
        [(A, A, 8, F32), (A + 28, A + 28, 8, F32)],                    # views that share an element
        [(A, A, 100, F32), (A + 8, A + 8, 2, F32)],                    # one inside the other
        [(A, A + 4096, 8, F32), (A + 64, A + 4096, 8, F32)],           # one destination for two
        [(A, A + 16, 8, F32)],                                         # shifted onto its own source
        [(A, A + 4096, 8, F32), (A + 4096, A + 8192, 8, F32)],         # a destination that another entry reads
        [(A, A, 8, F32), (A, A + 4096, 8, F32)],                       # scaled in place, and read for another copy
        [(A + 16 * i, A + 16 * i, 4, F32) for i in range(2000)] + [(A + 16 * 700 + 12, A + 16 * 700 + 12, 1, F32)],
        [(A, A, 8, BF16), (A + 8, A + 8, 1, F32)],
    ]
    for entries in refused:
        assert calls(*entries) == (INVALID, INVALID), entries[:3]
    # reading an element twice is no conflict: the norm alone, and copies into places of their own
    if not torch.cuda.is_available():                                  # (these would run)
        flat = (C.c_int64 * 8)(A, 0, 8, F32, A, 0, 8, F32)
        assert lib.hdqt_grad_norm(C.addressof(flat), 2, 2, 256, 256, 1 << 20, None) != INVALID
        for entries in ([(A, A, 8, F32), (A + 32, A + 32, 8, F32)], [(A, A, 8, F32), (A, A, 0, F32)],
                        [(A, A + 4096, 8, F32), (A, A + 8192, 8, F32)], [(A, A + 32, 8, F32), (A + 64, A + 96, 8, F32)],
                        [(A + 16 * i, A + 16 * i, 4, F32) for i in reversed(range(2000))]):
            assert INVALID not in calls(*entries)


@pytest.mark.parametrize("w_is_cd", [False, True])
def test_a_bias_of_another_type_or_size_is_named(plain_calls, w_is_cd):
    x, w = torch.randn(6, 4).bfloat16(), torch.randn((5, 4) if w_is_cd else (4, 5)).bfloat16()
    labels = torch.randint(0, 5, (6,))
    for bias in (torch.randn(5), torch.randn(5).half(), torch.randn(4).bfloat16(), torch.randn(5, 1).bfloat16()):
        with pytest.raises(ValueError, match="bias"):
            hnn.linear_cross_entropy(x, w, labels, bias=bias, w_is_cd=w_is_cd)
    got = hnn.linear_cross_entropy(x, w, labels, bias=torch.ones(5).bfloat16(), w_is_cd=w_is_cd)
    assert float(got) == pytest.approx(float(hnn.linear_cross_entropy(x, w, labels, w_is_cd=w_is_cd)), abs=1e-5)


def test_strides_of_images_without_pixels():
    """Any order of sizes with a 0 in it is an image without pixels, whatever torch writes down as its strides."""
    for shape in ((2, 3, 0, 8), (2, 0, 3, 8), (2, 0, 0, 8), (0, 3, 0, 8), (2, 0, 8), (1, 5, 3, 0, 8), (0, 3, 3, 8)):
        batch, pixel = hdqt._pixel_strides(torch.empty(shape), "x")
        assert pixel >= 8 and batch >= 0
    assert hdqt._pixel_strides(torch.empty(2, 5, 3, 8), "x") == (120, 8)
    assert hdqt._pixel_strides(torch.empty(2, 5, 3, 48)[..., :8], "x") == (720, 48)
    with pytest.raises(ValueError):
        hdqt._pixel_strides(torch.empty(2, 5, 3, 8)[:, :, ::2], "x")
    with pytest.raises(ValueError):
        hdqt._pixel_strides(torch.empty(2, 8, 3, 0).transpose(1, 3), "x")        # channels still have to be contiguous


def test_group_norm_module_names_groups_that_do_not_divide_the_channels():
    for channels, groups in ((48, 32), (8, 3), (8, 0), (8, -2)):
        with pytest.raises(ValueError, match="groups"):
            hnn.GroupNormAct(channels, groups=groups)
    with pytest.raises(ValueError, match="act"):
        hnn.GroupNormAct(8, groups=2, act="gelu")
    assert hnn.GroupNormAct(8).groups == 8 and hnn.GroupNormAct(64).groups == 32
