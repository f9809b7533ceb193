"""Linear layer + softmax cross entropy against 64-bit arithmetic.

Tolerances.  Sums of products are fp32 on the tensor cores, which may drop the bits below the accumulator's last place at each
addition of 16 products: at most 2^-23 of the running sum, which sum|x w| bounds.  With D features that is
  ez = (D/16 + 16) 2^-23 sum_d |x_d w_d|                     per logit (bf16; fp32 the same with parts of 64 additions)
  lse: ez averaged by the softmax + 2^-20 (fast exponential, 24-bit log)          loss: that + the label's ez
  dz : p (ez + e_lse) + 2^-20 p, and for bf16 one rounding 2^-8 |dz| and the code's 2^-12
  dX, dW: sums of |dz error| |w|, (K/16 + 16) 2^-23 sum |dz w|, one rounding to the type.
"""
import math

import pytest
import torch

from paper_2310_03675_b200 import hdqt

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def additions(k, dtype):
    return (min(k / 16, 64) + k / 1024 + 16 if dtype == torch.float32 else k / 16 + 16) * 2.0 ** -23


def reference(x, w, labels, weights, dtype, ignore=-100):
    """w [V, D] in 64 bits.  Values and error bounds of the docstring."""
    x, w = x.double(), w.double()
    v, d = w.shape
    t = x.shape[0]
    z = x @ w.t()
    ez = additions(d, dtype) * (x.abs() @ w.abs().t()) + (2.0 ** -22 * z.abs())
    kept = labels != ignore
    at = torch.where(kept, labels, 0)
    lse = torch.logsumexp(z, 1)
    p = torch.softmax(z, 1)
    e_lse = (p * ez).sum(1) + 2.0 ** -20 * (1 + lse.abs())
    loss = torch.where(kept, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    e_loss = torch.where(kept, e_lse + ez.gather(1, at[:, None])[:, 0] + 2.0 ** -22 * loss, 0.0)
    dz = p.clone()
    hot = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    gw = torch.where(kept, weights.double(), 0.0)[:, None]
    dz = (p - hot) * gw
    edz = gw.abs() * p * (ez + e_lse[:, None] + 2.0 ** -19)
    if dtype == torch.bfloat16:
        edz = edz + gw.abs() * (p * 2.0 ** -12 + 2.0 ** -32) + 2.0 ** -8 * dz.abs()
    else:
        edz = edz + 2.0 ** -23 * dz.abs()
    u = UNIT[dtype]

    def product(a, ea, b, k):
        val = a @ b
        err = ea @ b.abs() + (additions(k, dtype) + 2.0 ** -22) * (a.abs() @ b.abs())
        return val, err + u * (val.abs() + err)

    return {"lse": (lse, e_lse), "loss": (loss, e_loss), "dx": product(dz, edz, w, v),
            "dw": product(dz.t(), edz.t(), x, t)}


def close(got, want, name):
    value, err = want
    diff = (got.double() - value).abs()
    ok = diff <= err + 1e-37
    assert bool(ok.all()), (name, int((~ok).sum()), float((diff / (err + 1e-37)).max()))


def data(t, d, v, dtype, seed, scale=1.5, ignored=0.1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(t, d, generator=g, device="cuda").to(DT[dtype])
    w = (torch.randn(v, d, generator=g, device="cuda") * scale / math.sqrt(d)).to(DT[dtype])
    labels = torch.randint(0, v, (t,), generator=g, device="cuda")
    if ignored:
        labels[torch.rand(t, generator=g, device="cuda") < ignored] = -100
    weights = torch.rand(t, generator=g, device="cuda") - 0.3
    return x, w, labels, weights


SHAPES = [    # tokens, features, classes
    (1, 8, 3),
    (1, 64, 1),
    (3, 1, 5),
    (2, 17, 33),
    (128, 512, 100),
    (257, 72, 300),
    (130, 200, 1000),
    (512, 1000, 513),
    (31, 96, 5000),
    (700, 65, 2051),
    (1, 256, 20000),
    (1000, 8, 2),
    (512, 100, 300),
    (5, 100, 30001),
    (8, 2048, 3000),
    (2, 72, 9000),
    (20, 264, 6001),
    (32, 100, 7000),
    (4, 520, 9001),
    (120, 250, 260),
    (130, 16500, 300),
    (2500, 1600, 70),
]


@pytest.mark.gpu
@pytest.mark.parametrize("w_is_cd", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_all_calls_match_64_bits(case, dtype, w_is_cd):
    t, d, v = SHAPES[case]
    x, w, labels, weights = data(t, d, v, dtype, seed=case)
    ww = w if w_is_cd else w.t().contiguous()
    status = hdqt.new_status("cuda")
    kept = int((labels != -100).sum())
    for reduction in ("none", "mean", "sum"):
        if reduction == "mean" and kept == 0:
            continue
        gw = weights if reduction == "none" else torch.full_like(weights, 0.7 / kept if reduction == "mean" else 0.7)
        g = weights if reduction == "none" else torch.tensor(0.7, device="cuda")
        want = reference(x, w, labels, gw, DT[dtype])
        if reduction != "none":
            s = 1.0 / kept if reduction == "mean" else 1.0
            want["loss"] = (want["loss"][0].sum() * s, want["loss"][1].sum() * s + 2.0 ** -23 * want["loss"][0].sum().abs() * s)
        how = {"reduction": reduction, "w_is_cd": w_is_cd, "dev_status": status}
        loss, lse = hdqt.linear_xent_fwd(x, ww, labels, **how)
        close(loss, want["loss"], "loss")
        close(lse, want["lse"], "lse")
        dx, dw = hdqt.linear_xent_bwd(x, ww, labels, lse, g, **how)
        close(dx, want["dx"], "dx")
        close(dw if w_is_cd else dw.t(), want["dw"], "dw")
        loss2, lse2, dx2, dw2 = hdqt.linear_xent_train(x, ww, labels, g, **how)
        assert torch.equal(loss2, loss) or bool(((loss2 - loss).abs() <= 2.0 ** -20 * (1 + loss.abs())).all())
        close(lse2, want["lse"], "lse (train)")
        close(dx2, want["dx"], "dx (train)")
        close(dw2 if w_is_cd else dw2.t(), want["dw"], "dw (train)")
        # a stated piece size selects the tensor-core path whatever the size
        loss3, lse3, dx3, dw3 = hdqt.linear_xent_train(x, ww, labels, g, piece_bytes=1 << 28, **how)
        close(loss3, want["loss"], "loss (products)")
        close(lse3, want["lse"], "lse (products)")
        close(dx3, want["dx"], "dx (products)")
        close(dw3 if w_is_cd else dw3.t(), want["dw"], "dw (products)")
        dx4, dw4 = hdqt.linear_xent_bwd(x, ww, labels, lse, g, piece_bytes=1 << 28, **how)
        close(dx4, want["dx"], "dx (products, bwd)")
        close(dw4 if w_is_cd else dw4.t(), want["dw"], "dw (products, bwd)")
    hdqt.check_device_status(status)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pieces_give_the_same_result(dtype):
    """A small buffer cuts the tokens (training) or the vocabulary (backward) into pieces."""
    for w_is_cd in (True, False):
        x, w, labels, weights = data(900, 136, 1500, dtype, seed=3)
        ww = w if w_is_cd else w.t().contiguous()
        want = reference(x, w, labels, weights, DT[dtype])
        loss, lse = hdqt.linear_xent_fwd(x, ww, labels, reduction="none", w_is_cd=w_is_cd)
        for piece in (1, 1 << 20, 4 << 20):
            dx, dw = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, reduction="none", w_is_cd=w_is_cd, piece_bytes=piece)
            close(dx, want["dx"], "dx")
            close(dw if w_is_cd else dw.t(), want["dw"], "dw")
            _, _, dx, dw = hdqt.linear_xent_train(x, ww, labels, weights, reduction="none", w_is_cd=w_is_cd, piece_bytes=piece)
            close(dx, want["dx"], "dx (train)")
            close(dw if w_is_cd else dw.t(), want["dw"], "dw (train)")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pieces_whose_products_are_split_too(dtype):
    """Few tokens against many classes: dX has few blocks, so each piece of the vocabulary splits its share of the sum."""
    for w_is_cd, tokens in ((True, 300), (False, 150)):
        x, w, labels, weights = data(tokens, 64, 20011, dtype, seed=4)
        ww = w if w_is_cd else w.t().contiguous()
        want = reference(x, w, labels, weights, DT[dtype])
        loss, lse = hdqt.linear_xent_fwd(x, ww, labels, reduction="none", w_is_cd=w_is_cd)
        how = {"reduction": "none", "w_is_cd": w_is_cd}
        for classes in (10240, 7000, 20000):
            piece = tokens * classes * (2 if dtype == "bf16" else 6)
            dx, dw = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, piece_bytes=piece, **how)
            close(dx, want["dx"], "dx")
            close(dw if w_is_cd else dw.t(), want["dw"], "dw")
            dx, _ = hdqt.linear_xent_bwd(x, ww, labels, lse, weights, piece_bytes=piece, want_dw=False, **how)
            close(dx, want["dx"], "dx alone")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_strided_rows_odd_addresses_and_partial_gradients(dtype):
    t, d, v = 70, 48, 200
    wide_x, wide_w, labels, weights = data(t, d + 30, v, dtype, seed=5)
    wide_w = torch.cat([wide_w, wide_w])
    for off in (0, 8, 3):
        x, w = wide_x[:, off:off + d], wide_w[off:off + v, off:off + d]
        want = reference(x, w, labels, weights, DT[dtype])
        loss, lse, dx, dw = hdqt.linear_xent_train(x, w, labels, weights, reduction="none", w_is_cd=True)
        for got, name in ((loss, "loss"), (lse, "lse"), (dx, "dx"), (dw, "dw")):
            close(got, want[name], name)
        only = hdqt.linear_xent_train(x, w, labels, weights, reduction="none", w_is_cd=True, want_dw=False)
        assert only[3] is None
        close(only[2], want["dx"], "dx")
        only = hdqt.linear_xent_bwd(x, w, labels, lse, weights, reduction="none", w_is_cd=True, want_dx=False)
        assert only[0] is None
        close(only[1], want["dw"], "dw")


@pytest.mark.gpu
def test_large_logits_and_lowest_values():
    """Logits hundreds apart, and classes masked by the lowest bf16 value through a mask feature."""
    x, w, labels, weights = data(64, 32, 400, "bf16", seed=6, scale=60.0, ignored=0)
    want = reference(x, w, labels, weights, torch.bfloat16)
    loss, lse, dx, dw = hdqt.linear_xent_train(x, w, labels, weights, reduction="none", w_is_cd=True)
    for got, name in ((loss, "loss"), (lse, "lse"), (dx, "dx"), (dw, "dw")):
        close(got, want[name], name)
    x[:, 0] = 1.0
    w[:, 0] = 0.0
    w[100:, 0] = torch.finfo(torch.bfloat16).min           # classes that no token may take
    labels = labels % 100
    want = reference(x[:, 1:], w[:100, 1:], labels, weights, torch.bfloat16)
    loss, lse, dx, dw = hdqt.linear_xent_train(x, w, labels, weights, reduction="none", w_is_cd=True)
    assert float((lse.double() - want["lse"][0]).abs().max()) < 1e-3 * float(want["lse"][0].abs().max())
    assert not dw[100:].any()
    _, dw2 = hdqt.linear_xent_bwd(x, w, labels, lse, weights, reduction="none", w_is_cd=True)
    assert not dw2[100:].any()


@pytest.mark.gpu
def test_non_finite_inputs_stay_in_their_row():
    for dtype, piece in (("bf16", 0), ("fp32", 0), ("bf16", 1 << 28), ("fp32", 1 << 28)):
        x, w, labels, weights = data(40, 24, 300, dtype, seed=7, ignored=0)
        x[5, 3] = math.nan
        x[9, 2] = math.inf
        how = {"reduction": "none", "w_is_cd": True, "piece_bytes": piece}
        loss, lse, dx, dw = hdqt.linear_xent_train(x, w, labels, weights, **how)
        bad = torch.zeros(40, dtype=torch.bool, device="cuda")
        bad[5] = bad[9] = True
        assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(dx).all(1), bad)
        assert bool(torch.isnan(dw).all())
        labels[5] = labels[9] = -100          # an ignored row takes part in nothing but its own lse
        loss, lse, dx, dw = hdqt.linear_xent_train(x, w, labels, weights, **how)
        assert not bool(torch.isnan(loss).any()) and not bool(torch.isnan(dx).any())


@pytest.mark.gpu
def test_ignored_invalid_and_missing_tokens():
    x, w, labels, weights = data(50, 32, 90, "bf16", seed=8, ignored=0)
    none = torch.full_like(labels, -100)
    for piece in (0, 1 << 28):
        loss, lse, dx, dw = hdqt.linear_xent_train(x, w, none, w_is_cd=True, piece_bytes=piece)
        assert math.isnan(float(loss)) and not dx.any() and not dw.any()
        loss, _, dx, dw = hdqt.linear_xent_train(x, w, none, reduction="sum", w_is_cd=True, piece_bytes=piece)
        assert float(loss) == 0.0 and not dx.any() and not dw.any()
        status = hdqt.new_status("cuda")
        bad = labels.clone()
        bad[7], bad[8] = 90, -1
        loss, _, dx, dw = hdqt.linear_xent_train(x, w, bad, weights, reduction="none", w_is_cd=True, dev_status=status,
                                                 piece_bytes=piece)
        assert torch.equal(torch.isnan(loss).nonzero().flatten().cpu(), torch.tensor([7, 8]))
        assert not dx[7:9].any() and dx[6].any() and not bool(torch.isnan(dw).any())
        with pytest.raises(hdqt.HdqtError):
            hdqt.check_device_status(status)
    # a few tokens against a large vocabulary
    x, w, labels, _ = data(4, 64, 9000, "bf16", seed=11, ignored=0)
    status = hdqt.new_status("cuda")
    labels[1], labels[2] = -100, 9000
    loss, lse = hdqt.linear_xent_fwd(x, w, labels, reduction="none", w_is_cd=True, dev_status=status)
    assert float(loss[1]) == 0.0 and math.isnan(float(loss[2])) and bool(torch.isfinite(loss[[0, 3]]).all())
    with pytest.raises(hdqt.HdqtError):
        hdqt.check_device_status(status)
    assert math.isnan(float(hdqt.linear_xent_fwd(x, w, torch.full_like(labels, -100), w_is_cd=True)[0]))
    x, w, labels, weights = data(50, 32, 90, "bf16", seed=8, ignored=0)
    e = torch.empty(0, 32, device="cuda", dtype=torch.bfloat16)
    no = torch.empty(0, device="cuda", dtype=torch.int64)
    loss, lse, dx, dw = hdqt.linear_xent_train(e, w, no, w_is_cd=True)
    assert math.isnan(float(loss)) and lse.shape == (0,) and dx.shape == e.shape and not dw.any()
    dx, dw = hdqt.linear_xent_bwd(e, w, no, lse, w_is_cd=True)
    assert not dw.any()


@pytest.mark.gpu
def test_gradient_matches_differences():
    """<grad, v> against (L(+h v) - L(-h v)) / 2h in fp32 mode with h = 2^-6: the third-derivative term is h^2/6 |v|^3-sized
    (4e-5), the rounding of the two losses 2^-20 / h = 6e-5; L is a mean of O(1) terms."""
    x, w, labels, _ = data(60, 40, 150, "fp32", seed=9)
    _, _, dx, dw = hdqt.linear_xent_train(x, w, labels, w_is_cd=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    for which, grad in ((0, dx), (1, dw)):
        v = torch.randn((x, w)[which].shape, generator=g, device="cuda")
        v /= v.norm() / 4
        h, loss = 2.0 ** -6, []
        for sign in (1, -1):
            args = [x, w]
            args[which] = args[which] + sign * h * v
            loss.append(float(hdqt.linear_xent_fwd(*args, labels, w_is_cd=True)[0]))
        want = (loss[0] - loss[1]) / (2 * h)
        assert abs(float((grad.double() * v.double()).sum()) - want) <= 5e-4


@pytest.mark.gpu
def test_same_bits_again_and_on_another_stream():
    x, w, labels, weights = data(300, 128, 3000, "bf16", seed=10)
    first = hdqt.linear_xent_train(x, w, labels, w_is_cd=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = hdqt.linear_xent_train(x, w, labels, w_is_cd=True)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_refusals():
    import ctypes as C
    x, w = torch.zeros(4, 8), torch.zeros(8, 5)
    with pytest.raises(ValueError):
        hdqt.linear_xent_fwd(x, w, torch.zeros(4, dtype=torch.int64))           # not on a GPU
    lib = hdqt.lib
    INVALID, UNSUPPORTED, ALIGN, WS = 1, 2, 3, 4

    def desc(**over):
        d = hdqt.XentDesc(10, 16, 40, 16, 40, 16, 40, -100, 0, 1, 0, 1, 0)
        for k, v in over.items():
            setattr(d, k, v)
        return d

    def fwd(d, x=256, w=256, labels=256, loss=256, lse=256, ws=256, n=1 << 30):
        return lib.hdqt_linear_xent_fwd(C.byref(d), x, w, labels, loss, lse, ws, n, None, None)

    def bwd(d, lse=256, g=256, dx=256, dw=256, n=1 << 30):
        return lib.hdqt_linear_xent_bwd(C.byref(d), 256, 256, 256, lse, g, dx, dw, 256, n, None, None)

    for bad in ({"tokens": -1}, {"features": 0}, {"classes": 0}, {"ld_x": 15}, {"ld_w": 39}, {"reduction": 3},
                {"reduction": -1}, {"dtype": 9}, {"piece_bytes": -1}, {"w_is_cd": 1, "ld_w": 15}):
        assert fwd(desc(**bad)) == INVALID, bad
        assert lib.hdqt_linear_xent_workspace_bytes(C.byref(desc(**bad)), 0) == 0
    assert fwd(desc(dtype=2)) == UNSUPPORTED                                     # fp16
    assert fwd(desc(tokens=1 << 31)) == UNSUPPORTED
    for null in ("x", "w", "labels", "loss", "lse", "ws"):
        assert fwd(desc(), **{null: None}) == INVALID, null
    assert fwd(desc(), x=264) == ALIGN and fwd(desc(), w=258) == ALIGN and fwd(desc(), labels=260) == ALIGN
    assert fwd(desc(), ws=384) == ALIGN and fwd(desc(), loss=257) == ALIGN
    assert fwd(desc(dtype=0), x=258) == ALIGN
    assert fwd(desc(), n=64) == WS
    assert bwd(desc(ld_dx=15)) == INVALID and bwd(desc(ld_dw=39)) == INVALID
    assert bwd(desc(), lse=None) == INVALID and bwd(desc(reduction=0), g=None) == INVALID
    assert bwd(desc(), dx=257) == ALIGN and bwd(desc(), n=64) == WS
    assert lib.hdqt_linear_xent_train(C.byref(desc(reduction=0)), 256, 256, 256, None, 256, 256, 256, 256, 256, 1 << 30,
                                      None, None) == INVALID
    assert lib.hdqt_linear_xent_workspace_bytes(C.byref(desc()), 3) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [3, 20])
def test_weight_offsets_past_32_bits(tokens):
    """2.4e9 weights (and as many gradients): classes at both ends of the vocabulary, both ways of storing W."""
    d, v = 4096, 590_000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(tokens, d, generator=g, device="cuda").bfloat16()
    w = torch.empty((v, d), dtype=torch.bfloat16, device="cuda")
    for a in range(0, v, 59_000):
        w[a:a + 59_000] = torch.randn(min(59_000, v - a), d, generator=g, device="cuda") * (1.5 / math.sqrt(d))
    labels = torch.randint(0, v, (tokens,), generator=g, device="cuda")
    labels[0], labels[1] = v - 1, 0
    z = torch.cat([x.double() @ w[a:a + 59_000].double().t() for a in range(0, v, 59_000)], 1)
    lse = torch.logsumexp(z, 1)
    dz = torch.softmax(z, 1)
    dz[torch.arange(tokens), labels] -= 1
    for w_is_cd in (True, False):
        ww = w if w_is_cd else w.t().contiguous()
        loss, got_lse, dx, dw = hdqt.linear_xent_train(x, ww, labels, reduction="sum", w_is_cd=w_is_cd)
        assert float((got_lse.double() - lse).abs().max()) < 1e-4
        if not w_is_cd:
            dw = dw.t()
        for rows in (slice(0, 300), slice(v - 300, v)):
            want = dz[:, rows].t() @ x.double()
            far = (dw[rows].double() - want).abs()
            # dz and the result are rounded to bf16 (2^-8 each), sums of `tokens` terms
            assert bool((far <= 2.0 ** -6.5 * (dz[:, rows].abs().t() @ x.double().abs()) + 1e-30).all())
        want = torch.zeros(tokens, d, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(want)
        for a in range(0, v, 59_000):
            want += dz[:, a:a + 59_000] @ w[a:a + 59_000].double()
            size += dz[:, a:a + 59_000].abs() @ w[a:a + 59_000].double().abs()
        assert bool(((dx.double() - want).abs() <= 2.0 ** -7.5 * size).all())
        del ww, dw
