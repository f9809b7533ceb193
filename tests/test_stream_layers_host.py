"""Host side of the layer norm and dropout layers on the CPU: the library calls are replaced by plain torch.  Nothing is launched."""
import pytest
import torch

from paper_2310_03675_b200 import hdqt
from paper_2310_03675_b200 import nn as hnn


def mask(shape, p, seed, tag, offset):
    word = 0 if offset is None else int(offset)
    g = torch.Generator().manual_seed((seed * 1000003 + tag * 101 + word) % (1 << 62))
    return (torch.rand(shape, generator=g) >= p).float() / (1 - p if p < 1 else 1)


@pytest.fixture
def plain_calls(monkeypatch):
    def ln_fwd(x, gamma, beta, eps=1e-5, act="none"):
        with torch.no_grad():
            mean, var = x.mean(-1), x.var(-1, correction=0)
            rstd = (var + eps) ** -0.5
            z = (x - mean[..., None]) * rstd[..., None] * gamma + beta
            return torch.relu(z) if act == "relu" else z, mean, rstd

    def ln_bwd(dy, x, gamma, beta, mean, rstd, act="none", want_dx=True, want_params=True):
        with torch.enable_grad():
            ts = [t.detach().requires_grad_() for t in (x, gamma, beta)]
            y = torch.nn.functional.layer_norm(ts[0], x.shape[-1:], ts[1], ts[2])
            y = torch.relu(y) if act == "relu" else y
            dx, dg, db = torch.autograd.grad(y, ts, dy)
        return dx if want_dx else None, dg if want_params else None, db if want_params else None

    def drop(x, p, seed, tag=0, residual=None, philox_offset=None):
        with torch.no_grad():
            y = x * mask(x.shape, p, seed, tag, philox_offset) if p else x.clone()
            return y if residual is None else residual + y

    def dal_fwd(x, residual, gamma, beta, p, seed, tag=0, eps=1e-5, act="none", philox_offset=None):
        h = drop(x, p, seed, tag, residual, philox_offset)
        y, mean, rstd = ln_fwd(h, gamma, beta, eps, act)
        return y, h, mean, rstd

    def dal_bwd(dy, dh, h, gamma, beta, mean, rstd, p, seed, tag=0, act="none", philox_offset=None, want_dx=True, want_residual=True,
                want_params=True):
        g, dg, db = ln_bwd(dy, h, gamma, beta, mean, rstd, act, True, want_params)
        g = g if dh is None else g + dh
        return drop(g, p, seed, tag, None, philox_offset) if want_dx else None, g if want_residual else None, dg, db

    monkeypatch.setattr(hdqt, "layer_norm_fwd", ln_fwd)
    monkeypatch.setattr(hdqt, "layer_norm_bwd", ln_bwd)
    monkeypatch.setattr(hdqt, "dropout", drop)
    monkeypatch.setattr(hdqt, "dropout_add_layer_norm_fwd", dal_fwd)
    monkeypatch.setattr(hdqt, "dropout_add_layer_norm_bwd", dal_bwd)


def leaf(*shape):
    g = torch.Generator().manual_seed(sum(shape))
    return torch.randn(*shape, generator=g).requires_grad_()


@pytest.mark.parametrize("p", [0.0, 0.5])
@pytest.mark.parametrize("used", ["y", "h", "both"])
@pytest.mark.parametrize("needs", ["x", "residual", "x and residual"])
def test_gradients_of_the_fused_layer(plain_calls, p, used, needs):
    layer = hnn.DropoutAddLayerNorm(12, p, layer_id=2, act="relu")
    layer.step = 4
    x, r, cy, ch = leaf(5, 12), leaf(6, 12)[:5].detach().requires_grad_(), leaf(7, 12)[:5].detach(), leaf(8, 12)[:5].detach()
    x.requires_grad_("x" in needs.split()), r.requires_grad_("residual" in needs)
    y, h = layer(x, r)
    m = mask((5, 12), p, 4, 22, None) if p else torch.ones(5, 12)
    h2 = r + x * m
    y2 = torch.relu(torch.nn.functional.layer_norm(h2, (12,), layer.weight, layer.bias))
    leaves = [t for t in (x, r, layer.weight, layer.bias) if t.requires_grad]
    pick = lambda y, h: {"y": (y * cy).sum(), "h": (h * ch).sum(), "both": (y * cy).sum() + (h * ch).sum()}[used]  # noqa: E731
    got = torch.autograd.grad(pick(y, h), leaves, allow_unused=True)
    want = torch.autograd.grad(pick(y2, h2), leaves, allow_unused=True)
    for a, b in zip(got, want):
        assert (a is None) == (b is None)
        if a is not None:
            torch.testing.assert_close(a, b, rtol=1e-5, atol=1e-6)


def test_dropout_layer(plain_calls):
    drop = hnn.Dropout(0.5, layer_id=1)
    drop.step = 9
    x, r = leaf(4, 6), leaf(4, 6)
    y = drop(x, r)
    m = mask((4, 6), 0.5, 9, 14, None)
    torch.testing.assert_close(y, r + x * m)
    dx, dr = torch.autograd.grad(y.sum(), (x, r))
    torch.testing.assert_close(dx, m)
    torch.testing.assert_close(dr, torch.ones(4, 6))
    drop.eval()
    assert drop(x) is x and torch.equal(drop(x, r), x + r)


def test_second_derivatives_are_refused_where_there_are_none(plain_calls):
    x = leaf(3, 8)
    for layer in (hnn.LayerNormAct(8), lambda t: hnn.DropoutAddLayerNorm(8, 0.0)(t)[0]):
        g, = torch.autograd.grad(layer(x).pow(2).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(g.sum(), x)


def test_changed_device_word_is_reported(plain_calls):
    word = torch.zeros(1, dtype=torch.int32)
    y = hnn.Dropout(0.5, philox_offset=word)(leaf(4, 4))
    word += 1
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_mlp_options(plain_calls):
    with pytest.raises(ValueError):
        hnn.Mlp(norm="batch")
    with pytest.raises(ValueError):
        hnn.Mlp(residual=True)
    assert list(hnn.Mlp().state_dict()) == [f"layers.{i}.{k}" for i in range(3) for k in ("weight", "bias")]
    model = hnn.Mlp((10, 8, 8, 3), quantized=False, norm="layer", dropout=0.5, residual=True)
    kinds = [type(m) for m in model.norms]
    assert kinds == [hnn.LayerNormAct, hnn.DropoutAddLayerNorm]
    model.set_step(7)
    assert {m.step for m in model.modules() if isinstance(m, hnn._RANDOM)} == {7}
    x = leaf(5, 10)
    assert torch.equal(model(x), model(x))                    # one step, one mask
    a = model(x)
    model.set_step(8)
    assert not torch.equal(a, model(x))
    model(x).sum().backward()
    assert all(p.grad is not None for p in model.parameters())


def test_evenly_spaced_rows():
    t = torch.zeros(4, 6, 10)
    stride = lambda v: hdqt._row_stride(v, "x")  # noqa: E731
    assert stride(t) == 10 and stride(t[..., 2:5]) == 10 and stride(t[:, 3]) == 60 and stride(t[::2, 3]) == 120
    assert stride(t[0, 0]) == 10 and stride(t[:1, :1, :3]) == 3 and stride(t[:0]) == 10 and stride(t[0, 0, 0:1]) == 1
    for bad in (t[:, ::4], t.transpose(0, 1), t.transpose(1, 2), t[0, 0].expand(3, 10), t[:, :1].expand(4, 6, 10), torch.zeros(())):
        with pytest.raises(ValueError):
            stride(bad)
