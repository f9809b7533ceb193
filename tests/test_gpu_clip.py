"""Global gradient norm and clipping over lists of tensors against 64-bit arithmetic.

Tolerances: a per-thread fp32 sum of n squares is off by at most n 2^-24 relative (all terms are positive), and the
largest list here gives a thread fewer than 256 of them; the joins are fp64; the square root halves the relative error and
the result is rounded once: 256 / 2 * 2^-24 + 2^-24 < 2^-16.  A scaled element is off by that (the factor), one product
rounding and the rounding to its type (2^-24, 2^-8, 2^-11, or half the smallest subnormal of fp16).
"""
import math

import numpy as np
import pytest
import torch

from paper_2310_03675_b200 import hdqt

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a unit in the last place
NORM_RTOL = 2.0 ** -16


def _lists(sizes, kinds, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale).to(DT[k]) for n, k in zip(sizes, kinds)]


def _want_norm(ts, kind):
    if kind == 2.0:
        return math.sqrt(sum(float(t.double().square().sum()) for t in ts))
    return max([float(t.double().abs().max()) for t in ts if t.numel()] + [0.0])


def _check_scaled(got, src, factor):
    for a, b in zip(got, src):
        want = b.double() * factor
        tol = want.abs() * (NORM_RTOL + 2.0 ** -23 + UNIT[b.dtype]) + (2.0 ** -25 if b.dtype == torch.float16 else 1e-44)
        assert bool(((a.double() - want).abs() <= tol).all())


CASES = [
    ([1], ["fp32"]),
    ([0, 5, 0, 1], ["fp32", "bf16", "fp16", "fp32"]),
    ([1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33], ["bf16"] * 11),
    ([8191, 8192, 8193, 16383, 16384, 16385, 100001], ["fp32", "fp16", "bf16", "fp32", "bf16", "fp16", "fp32"]),
    ([37] * 64, ["fp32"] * 64),
    ([41] * 65, ["bf16"] * 65),
    ([3 + i % 11 for i in range(1100)], [("fp32", "bf16", "fp16")[i % 3] for i in range(1100)]),   # several tables
    ([2_000_003, 5], ["fp32", "bf16"]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("norm_type", [2.0, math.inf])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_norm_and_clipping_match_64_bits(case, norm_type):
    sizes, kinds = CASES[case]
    ts = _lists(sizes, kinds, seed=case)
    want = _want_norm(ts, norm_type)
    rtol = NORM_RTOL if norm_type == 2.0 else 0.0
    norm = hdqt.grad_norm(ts, norm_type)
    assert norm.dtype == torch.float32 and norm.shape == ()
    assert abs(float(norm) - want) <= rtol * want
    for max_norm in (0.3 * want, 2.0 * want + 1.0, 0.0):
        factor = min(1.0, max_norm / (want + 1e-6))
        out = [torch.full_like(t, 7) for t in ts]
        before = [t.clone() for t in ts]
        n2 = hdqt.clip_grad_norm(ts, max_norm, norm_type, out=out)
        assert float(n2) == float(norm)
        assert all(torch.equal(a, b) for a, b in zip(ts, before))          # sources are left alone
        _check_scaled(out, ts, factor)
        inplace = [t.clone() for t in ts]
        hdqt.clip_grad_norm(inplace, max_norm, norm_type)
        assert all(torch.equal(a, b) for a, b in zip(inplace, out))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shift", [1, 2, 3, 5])
def test_any_element_alignment(kind, shift):
    base = _lists([5000 + shift], [kind], seed=shift)[0]
    ts = [base[shift:4000], base[4000:]]                # odd starting addresses, one buffer
    want = _want_norm(ts, 2.0)
    out = [torch.empty_like(t) for t in ts]             # other alignment than the sources
    assert abs(float(hdqt.clip_grad_norm(ts, 0.5, out=out)) - want) <= NORM_RTOL * want
    _check_scaled(out, ts, 0.5 / (want + 1e-6))
    guard = base.clone()
    hdqt.clip_grad_norm(ts, 0.5)
    assert torch.equal(base[:shift], guard[:shift])     # nothing beside the tensors is written
    assert all(torch.equal(a, b) for a, b in zip(ts, out))


@pytest.mark.gpu
def test_nothing_to_do_and_non_finite_values():
    assert float(hdqt.grad_norm([], device="cuda")) == 0.0
    assert float(hdqt.clip_grad_norm([], 1.0, device="cuda")) == 0.0
    assert float(hdqt.clip_grad_norm([torch.zeros(0, device="cuda")], 1.0)) == 0.0
    z = torch.zeros(100, device="cuda")
    assert float(hdqt.clip_grad_norm([z], 1.0)) == 0.0 and not z.any()
    for norm_type in (2.0, math.inf):
        t = [torch.ones(50, device="cuda"), torch.ones(3, device="cuda", dtype=torch.bfloat16)]
        t[1][2] = math.nan
        assert math.isnan(float(hdqt.clip_grad_norm(t, 1.0, norm_type)))
        assert all(bool(torch.isnan(x).all()) for x in t)
        t = [torch.ones(50, device="cuda"), torch.tensor([2.0, -math.inf], device="cuda")]
        assert float(hdqt.clip_grad_norm(t, 1.0, norm_type)) == math.inf
        assert not t[0].any() and float(t[1][0]) == 0.0 and math.isnan(float(t[1][1]))


@pytest.mark.gpu
def test_same_bits_again_and_on_another_stream():
    ts = _lists([300_007, 12, 70_001], ["fp32", "bf16", "fp16"], seed=5)
    norm = hdqt.grad_norm(ts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = [torch.empty_like(t) for t in ts]
        again = [hdqt.clip_grad_norm(ts, 1.0, out=out) for _ in range(5)]
    side.synchronize()
    assert all(float(a) == float(norm) for a in again)


@pytest.mark.gpu
def test_scaling_by_a_device_scalar():
    ts = _lists([1, 100, 70_001, 33], ["fp32", "bf16", "fp16", "fp32"], seed=6)
    for f in (0.37, -3.0, 1.0, 0.0):
        factor = torch.tensor(f, device="cuda")
        out = [torch.full_like(t, 5) for t in ts]
        hdqt.scale_tensors(ts, factor, out=out)
        want = [(t.float() * factor).to(t.dtype) for t in ts]           # one product, one rounding
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        inplace = [t.clone() for t in ts]
        hdqt.scale_tensors(inplace, factor)
        assert all(torch.equal(a, b) for a, b in zip(inplace, want))
    hdqt.scale_tensors([], factor)
    with pytest.raises(ValueError):
        hdqt.scale_tensors(ts, torch.ones(2, device="cuda"))


def test_refusals():
    ok = torch.zeros(4)
    with pytest.raises(ValueError):
        hdqt.grad_norm([ok])                              # not on a GPU
    with pytest.raises(ValueError):
        hdqt.grad_norm([ok], norm_type=1.0)
    lib = hdqt.lib
    INVALID, ALIGN, WS = 1, 3, 4
    import ctypes as C

    def call(entry, norm_type=2, max_norm=1.0, norm_out=256, ws=256, ws_bytes=1 << 20, count=1):
        table = (C.c_int64 * 4)(*entry)
        return lib.hdqt_clip_grad_norm(C.addressof(table), count, norm_type, max_norm, norm_out, ws, ws_bytes, None)

    assert call((256, 256, 8, 3)) == INVALID              # unknown type
    assert call((256, 256, -1, 0)) == INVALID
    assert call((0, 256, 8, 0)) == INVALID
    assert call((256, 0, 8, 0)) == INVALID
    assert call((256, 256, 8, 0), norm_type=1) == INVALID
    assert call((256, 256, 8, 0), max_norm=-1.0) == INVALID
    assert call((256, 256, 8, 0), max_norm=math.nan) == INVALID
    assert call((256, 256, 8, 0), norm_out=None) == INVALID
    assert call((256, 256, 8, 0), count=-1) == INVALID
    assert call((258, 256, 8, 0)) == ALIGN
    assert call((256, 257, 8, 1)) == ALIGN
    assert call((256, 256, 8, 0), ws=320 + 8) == ALIGN
    assert call((256, 256, 8, 0), ws_bytes=16) == WS
    assert lib.hdqt_grad_norm(None, 2, 2, 256, 256, 1 << 20, None) == INVALID
    assert lib.hdqt_grad_norm_workspace_bytes(0) > 0
    table = (C.c_int64 * 4)(256, 256, 8, 0)
    assert lib.hdqt_scale_tensors(C.addressof(table), 1, None, None) == INVALID
    assert lib.hdqt_scale_tensors(C.addressof(table), 1, 258, None) == ALIGN
    assert lib.hdqt_scale_tensors(C.addressof(table), -1, 256, None) == INVALID


@pytest.mark.gpu
def test_offsets_past_32_bits():
    n = (1 << 31) + 12345
    big = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    tail = torch.full((3,), 2.0, device="cuda")
    norm = hdqt.clip_grad_norm([big, tail], 1.0)
    want = math.sqrt(n + 12.0)
    # a thread adds 7100 ones in fp32, exactly
    assert abs(float(norm) - want) <= 2.0 ** -22 * want
    f = torch.tensor(1.0 / (want + 1e-6)).to(torch.bfloat16)
    assert float(big[0]) == float(f) and float(big[-1]) == float(f) and bool((big[1 << 31:] == big[0]).all())
