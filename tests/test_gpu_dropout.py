"""Dropout from the counter-based generator against the oracle's random numbers and plain fp32 arithmetic: one multiplication, one
addition, one rounding, so that results are equal bit for bit."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import hdqt_oracle as O
from paper_2310_03675_b200 import hdqt
from paper_2310_03675_b200 import nn as hnn

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def kept(n, p, seed, tag=0, offset=0):
    """Which of n elements stay, from the oracle's generator."""
    g = np.arange((n + 7) // 8, dtype=np.uint64)
    w = O.philox4x32_10(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.full_like(g, tag), np.full_like(g, offset),
                        seed & 0xFFFFFFFF, seed >> 32)
    w = np.stack([np.asarray(v, dtype=np.uint64) for v in w], 1)
    u = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 2).reshape(-1)[:n]
    return torch.from_numpy(u >= np.uint64(round(p * 65536)))


def plain(x, p, keep, residual=None):
    t = round(p * 65536)
    scale = torch.tensor(65536 / (65536 - t) if t < 65536 else 0.0, dtype=torch.float32, device=x.device)
    d = torch.where(keep.view(x.shape), x.float() * scale, 0.0)
    return (d if residual is None else residual.float() + d).to(x.dtype)


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (4, 8), (33, 777), (1, 4096), (128, 2, 40), (1000, 1001), ()], ids=str)
def test_matches_the_oracle(shape, dtype):
    n = math.prod(shape)
    for p, seed, tag, word in ((0.1, 0, 0, None), (0.5, 1, 6, 3), (0.999, (1 << 64) - 1, (1 << 32) - 1, -1), (1 / 3, 1 << 40, 14, 9)):
        offset = None if word is None else torch.tensor([word], dtype=torch.int32, device="cuda")
        keep = kept(n, p, seed, tag, 0 if word is None else word & 0xFFFFFFFF).cuda()
        x, res = normal(shape, dtype, 1), normal(shape, dtype, 2)
        for r in (None, res):
            y = hdqt.dropout(x, p, seed, tag, r, offset)
            assert y.shape == x.shape and y.dtype == x.dtype and torch.equal(y, plain(x, p, keep, r))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_probabilities_at_the_ends_and_garbage_in_dropped_places(dtype):
    x, res = normal((37, 64), dtype, 1), normal((37, 64), dtype, 2)
    for p in (0.0, 2.0 ** -18):                      # nothing is dropped
        assert torch.equal(hdqt.dropout(x, p, 1), x)
        assert torch.equal(hdqt.dropout(x, p, 1, residual=res), (res.float() + x.float()).to(x.dtype))
    for p in (1.0, 1.0 - 2.0 ** -18):                # everything is
        assert not hdqt.dropout(torch.full_like(x, math.nan), p, 1).any()
        assert torch.equal(hdqt.dropout(torch.full_like(x, math.inf), p, 1, residual=res), res)
    keep = kept(x.numel(), 0.5, 1).cuda().view(x.shape)
    for value in (math.nan, math.inf, -math.inf):
        assert torch.equal(hdqt.dropout(torch.where(keep, x, value), 0.5, 1, residual=res), hdqt.dropout(x, 0.5, 1, residual=res))
    assert bool(torch.isnan(hdqt.dropout(torch.full_like(x, math.nan), 0.5, 1)[keep]).all())


@pytest.mark.gpu
def test_share_of_kept_elements_and_independent_streams():
    """2^22 draws: the share kept is within 5 standard deviations of 1 - p, and two streams agree as often as independent ones."""
    n = 1 << 22
    x = torch.ones(n, device="cuda")
    a, b, c = hdqt.dropout(x, 0.25, 1), hdqt.dropout(x, 0.25, 1, tag=8), hdqt.dropout(x, 0.25, 2)
    for y in (a, b, c):
        share = float((y != 0).double().mean())
        assert abs(share - 0.75) < 5 * math.sqrt(0.25 * 0.75 / n)
        assert abs(float(y.double().mean()) - 1.0) < 5 * math.sqrt(0.25 / 0.75 / n)      # unbiased
    for u, v in ((a, b), (a, c), (b, c)):
        same = float(((u != 0) == (v != 0)).double().mean())
        q = 0.75 ** 2 + 0.25 ** 2
        assert abs(same - q) < 5 * math.sqrt(q * (1 - q) / n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_strides_and_addresses(dtype):
    wide, other = normal((5, 6, 100), dtype, 1), normal((5, 6, 100), dtype, 2)
    for lo, hi in ((0, 16), (8, 96), (3, 20), (99, 100), (0, 100), (1, 9)):
        x, r = wide[..., lo:hi], other[..., lo:hi]
        keep = kept(x.numel(), 0.3, 4).cuda()
        for res in (None, r, r.contiguous()):
            assert torch.equal(hdqt.dropout(x, 0.3, 4, residual=res), plain(x, 0.3, keep, res))
        assert torch.equal(hdqt.dropout(x.contiguous(), 0.3, 4, residual=r), plain(x, 0.3, keep, r))
    flat = wide.view(-1)
    for start in (1, 3, 4, 8):                       # dense, but starting anywhere
        x = flat[start:start + 999]
        assert torch.equal(hdqt.dropout(x, 0.3, 4), plain(x, 0.3, kept(999, 0.3, 4).cuda()))
    assert hdqt.dropout(wide[:0], 0.3, 4).shape == (0, 6, 100) and hdqt.dropout(wide[..., :0], 0.3, 4).shape == (5, 6, 0)
    with pytest.raises(ValueError):
        hdqt.dropout(wide[:, ::4], 0.3, 4)
    with pytest.raises(ValueError):
        hdqt.dropout(wide[0, :1].expand(4, 100), 0.3, 4)
    with pytest.raises(ValueError):
        hdqt.dropout(wide[0].t(), 0.3, 4)


@pytest.mark.gpu
def test_argument_checks():
    x = normal((4, 32), "bf16", 1)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    for i, call in enumerate([
            lambda: hdqt.dropout(x.double(), 0.1, 1), lambda: hdqt.dropout(x.cpu(), 0.1, 1), lambda: hdqt.dropout(x, 1.1, 1),
            lambda: hdqt.dropout(x, -0.1, 1), lambda: hdqt.dropout(x, math.nan, 1), lambda: hdqt.dropout(x, 0.1, -1),
            lambda: hdqt.dropout(x, 0.1, 1 << 64), lambda: hdqt.dropout(x, 0.1, 1, tag=-1),
            lambda: hdqt.dropout(x, 0.1, 1, residual=x.float()), lambda: hdqt.dropout(x, 0.1, 1, residual=x[:2]),
            lambda: hdqt.dropout(x, 0.1, 1, residual=x.cpu()), lambda: hdqt.dropout(x, 0.1, 1, philox_offset=word.cpu()),
            lambda: hdqt.dropout(x, 0.1, 1, philox_offset=word.long()), lambda: hdqt.dropout(x, 0.1, 1, philox_offset=word[:0]),
            lambda: hnn.Dropout(1.5), lambda: hnn.DropoutAddLayerNorm(8, -0.5), lambda: hnn.DropoutAddLayerNorm(8, 0.5, act="tanh")]):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} went through")


@pytest.mark.gpu
def test_more_than_2_to_the_31_elements():
    n = (1 << 31) + 4099
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = hdqt.dropout(x, 0.5, 21, tag=6)
    i = np.arange(n - 5000, n, dtype=np.uint64)
    g = i // np.uint64(8)
    w = O.philox4x32_10(g, np.zeros_like(g), np.full_like(g, 6), np.zeros_like(g), 21, 0)
    w = np.stack([np.asarray(v, dtype=np.uint64) for v in w], 1)
    j = (i % np.uint64(8)).astype(np.int64)
    word = w[np.arange(len(i)), j // 2]
    u = np.where(j % 2 == 0, word & np.uint64(0xFFFF), word >> np.uint64(16))
    assert torch.equal(y[-5000:].cpu() != 0, torch.from_numpy(u >= np.uint64(32768)))
    assert torch.equal(y[:4096].cpu() != 0, kept(4096, 0.5, 21, 6))


def test_refusals():
    with pytest.raises(ValueError):
        hdqt.dropout(torch.zeros(2, 8), 0.5, 1)                                # not on a GPU
    lib = hdqt.lib
    INVALID, UNSUPPORTED, ALIGN = 1, 2, 3

    def call(x=256, res=256, y=256, **over):
        d = hdqt.DropoutDesc(9, 16, 16, 16, 16, 0.5, 7, None, 3, 0)
        for k, v in over.items():
            setattr(d, k, v)
        return lib.hdqt_dropout_add(C.byref(d), x, res, y, None)

    for bad in ({"rows": -1}, {"cols": -1}, {"p": -0.1}, {"p": 1.1}, {"p": math.nan}, {"dtype": 5}, {"x_row_stride": 15},
                {"r_row_stride": 15}, {"y_row_stride": 15}, {"x": None}, {"y": None}):
        assert call(**bad) == INVALID, bad
    assert lib.hdqt_dropout_add(None, 256, 256, 256, None) == INVALID
    assert call(rows=1 << 30, cols=1 << 30, x_row_stride=1 << 30, y_row_stride=1 << 30, r_row_stride=1 << 30) == UNSUPPORTED
    for bad in ({"x": 258}, {"res": 257}, {"y": 258}, {"philox_offset": 258}):
        assert call(**bad) == ALIGN, bad
    assert call(x=None, y=None, rows=0) == 0 and call(x=None, y=None, cols=0) == 0
