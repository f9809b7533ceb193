"""Layer norm, dropout and both on the residual stream as layers: through autograd, in the quantized network, replayed from graphs."""
import pytest
import torch

from paper_2310_03675_b200 import hdqt
from paper_2310_03675_b200 import nn as hnn


def leaf(shape, seed, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype).requires_grad_()


@pytest.mark.gpu
def test_layers_have_the_gradients_of_their_calls():
    x, res = leaf((6, 9, 40), 1), leaf((6, 9, 40), 2)
    dy, dh = leaf((6, 9, 40), 3).detach(), leaf((6, 9, 40), 4).detach()
    norm = hnn.LayerNormAct(40, act="silu").cuda()
    norm(x).backward(dy)
    y, mean, rstd = hdqt.layer_norm_fwd(x.detach(), norm.weight.detach(), norm.bias.detach(), 1e-5, "silu")
    want = hdqt.layer_norm_bwd(dy, x.detach(), norm.weight.detach(), norm.bias.detach(), mean, rstd, "silu")
    assert all(torch.equal(a, b) for a, b in zip((x.grad, norm.weight.grad, norm.bias.grad), want))

    drop = hnn.Dropout(0.4, layer_id=3)
    drop.step = 17
    x.grad = None
    y = drop(x, res)
    assert torch.equal(y, hdqt.dropout(x.detach(), 0.4, 17, 8 * 3 + 6, res.detach()))
    y.backward(dy)
    assert torch.equal(x.grad, hdqt.dropout(dy, 0.4, 17, 30)) and torch.equal(res.grad, dy)
    g, = torch.autograd.grad(drop(x).pow(2).sum(), x, create_graph=True)       # dropout is linear: second derivatives are its own
    gg, = torch.autograd.grad(g.sum(), x)
    keep = (hdqt.dropout(torch.ones_like(dy), 0.4, 17, 30))
    assert torch.equal(gg, 2 * keep * keep)

    both = hnn.DropoutAddLayerNorm(40, 0.4, layer_id=3, act="silu").cuda()
    both.step = 17
    for used in ("y", "h", "both"):
        for t in (x, res, *both.parameters()):
            t.grad = None
        y, h = both(x, res)
        outs, grads = {"y": ([y], [dy]), "h": ([h], [dh]), "both": ([y, h], [dy, dh])}[used]
        torch.autograd.backward(outs, grads)
        if used == "h":
            assert torch.equal(res.grad, dh) and torch.equal(x.grad, hdqt.dropout(dh, 0.4, 17, 30)) and both.weight.grad is None
            continue
        _, hh, mean, rstd = hdqt.dropout_add_layer_norm_fwd(x.detach(), res.detach(), both.weight.detach(), both.bias.detach(), 0.4, 17,
                                                            30, act="silu")
        want = hdqt.dropout_add_layer_norm_bwd(dy, dh if used == "both" else None, hh, both.weight.detach(), both.bias.detach(), mean,
                                               rstd, 0.4, 17, 30, act="silu")
        assert all(torch.equal(a, b) for a, b in zip((x.grad, res.grad, both.weight.grad, both.bias.grad), want))
    both.eval(), drop.eval()
    for t in (x, res):
        t.grad = None
    y, h = both(x, res)
    assert torch.equal(h, x + res)
    torch.autograd.backward([y, h], [dy, dh])
    assert torch.equal(x.grad, res.grad) and x.grad.data_ptr() != res.grad.data_ptr()
    assert drop(x) is x
    y, h = both(x)
    assert torch.equal(h, x)
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad(both(x, res)[0].sum(), x, create_graph=True)
        torch.autograd.grad(g.sum(), x)


@pytest.mark.gpu
def test_layers_take_any_layout_and_16_bit_activations():
    norm, both = hnn.LayerNormAct(24).cuda(), hnn.DropoutAddLayerNorm(24, 0.0).cuda()
    x = leaf((24, 5, 7), 1, torch.bfloat16)
    t = x.permute(1, 2, 0)
    y = norm(t)
    assert y.dtype == torch.bfloat16 and torch.equal(y, norm(t.contiguous())) and torch.equal(y, both(t)[0])
    y.sum().backward()                                                          # (the incoming gradient is an expanded scalar)
    assert x.grad.shape == x.shape and norm.weight.grad.dtype == torch.float32
    assert torch.equal(hnn.Dropout(0.5)(t, t).shape == t.shape and t, t)


@pytest.mark.gpu
def test_seeds_come_from_torch_without_a_training_loop():
    drop, x = hnn.Dropout(0.5), torch.ones(4096, device="cuda")
    torch.manual_seed(1)
    a, b = drop(x), drop(x)
    torch.manual_seed(1)
    assert torch.equal(drop(x), a) and not torch.equal(a, b)


@pytest.mark.gpu
def test_a_changed_device_word_between_the_passes_is_an_error():
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = leaf((8, 16), 1)
    for layer in (hnn.Dropout(0.5, philox_offset=word), hnn.DropoutAddLayerNorm(16, 0.5, philox_offset=word).cuda()):
        y = layer(x)
        y = y if isinstance(y, torch.Tensor) else y[0]
        word += 1
        with pytest.raises(RuntimeError):
            y.sum().backward()


def mlp(**how):
    torch.manual_seed(0)
    return hnn.Mlp(sizes=(96, 64, 64, 12), norm="layer", dropout=0.25, residual=True, **how).cuda()


@pytest.mark.gpu
def test_network_of_quantized_products_with_all_of_them():
    """One step of the network against the same calls written out, gradients bit for bit."""
    model = mlp()
    x, labels = hnn.sensor_window_batch(50, 96, 12, seed=1, device="cuda")
    opt = torch.optim.SGD(model.parameters(), lr=0.0)
    loss = hnn.train_step(model, opt, x, labels, step=5)
    got = {k: p.grad.clone() for k, p in model.named_parameters()}
    l0, l1, l2 = model.layers
    n0, n1 = model.norms
    assert isinstance(n0, hnn.LayerNormAct) and isinstance(n1, hnn.DropoutAddLayerNorm)
    for p in model.parameters():
        p.grad = None
    a = hnn.LayerNormFunction.apply(l0(x), n0.weight, n0.bias, 1e-5, "relu")
    a = hnn.DropoutFunction.apply(a, None, 0.25, 5, 6, None)
    b, _ = hnn.DropoutAddLayerNormFunction.apply(l1(a), a, n1.weight, n1.bias, 0.25, 5, 14, None, 1e-5, "relu")
    again = torch.nn.functional.cross_entropy(l2(b), labels)
    again.backward()
    assert torch.equal(loss, again)
    assert all(torch.equal(p.grad, got[k]) for k, p in model.named_parameters())
    model.eval()
    assert torch.equal(model(x), model(x))


@pytest.mark.gpu
def test_recorded_steps_equal_eager_steps_and_drop_anew():
    x, labels = hnn.sensor_window_batch(64, 96, 12, seed=1, device="cuda")
    results = []
    for graphed in (False, True):
        model = mlp()
        opt = torch.optim.SGD(model.parameters(), lr=0.01, momentum=0.9)
        if graphed:
            step = hnn.GraphedTrainStep(model, opt, x, labels, base_step=3, clip_norm=1.0)
            word = step.counter
            losses = [float(step(x, labels).detach()) for _ in range(5)]
            assert int(word) == 8
        else:
            word = torch.zeros(1, dtype=torch.int32, device="cuda")
            for m in model.modules():
                if isinstance(m, hnn._RANDOM):
                    m.over = dict(m.over, philox_offset=word)
            model.set_step(3)
            losses = []
            for _ in range(8):
                opt.zero_grad(set_to_none=True)
                loss = torch.nn.functional.cross_entropy(model(x), labels)
                loss.backward()
                hnn.clip_grad_norm_(model.parameters(), 1.0)
                opt.step()
                word += 1
                losses.append(float(loss.detach()))
            losses = losses[3:]
        results.append((losses, [p.detach().clone() for p in model.parameters()]))
    assert results[0][0] == results[1][0]
    assert all(torch.equal(a, b) for a, b in zip(results[0][1], results[1][1]))
