"""GPU: slimfit_gated_quant_pack / slimfit_gated_backward_dequant against the formulas in 64 bits, at the tolerances the
header states; codes and scales are those of quant_pack bit for bit."""
import math

import numpy as np
import pytest
import torch

from oracle import ref
from paper_2305_18513_amd import autograd as ag
from paper_2305_18513_amd import binding as sf
from tests.gpu_util import Guarded, require_gpu, to_np

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _parts(g, act):
    """(act(g), act'(g)) in 64 bits."""
    if act == sf.ACT_SILU:
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    p = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def _near(got, want, tol, bf16):
    """|got - want| <= tol, plus half a step of bf16 (2^-8 of the value) and the smallest numbers."""
    tol = tol + 1e-37 + (want.abs() * 2.0 ** -8 if bf16 else 0.0)
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), "max excess %.3g" % float((off - tol).max())


def _input(rows, F, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, 2 * F, generator=g, device="cuda") * 2
    x.view(-1)[::17] *= 20.0
    x.view(-1)[::29] = 0.0
    x[0, :8] = torch.tensor([-90.0, 90.0, -300.0, 300.0, -0.0, 1e-30, -17.5, 3e4], device="cuda")
    return x.to(dtype), torch.randn(rows, F, generator=g, device="cuda").to(dtype)


def _run(x, dy, act, mode, bits, block, fb):
    rows, F = dy.shape
    n = x.numel()
    bf16 = x.dtype == torch.bfloat16
    blocked = mode == sf.Q_BLOCK
    codes, scales = Guarded(sf.packed_bytes(n, bits), torch.uint8), Guarded(sf.num_blocks(n, block) if blocked else 0, torch.float32)
    y, dx = Guarded(rows * F, x.dtype), Guarded(n, x.dtype)
    sc = scales.t if blocked else None
    sf.gated_quant_pack(x, act, mode, bits, block, fb, y.t.view(rows, F), codes.t if bits else None, sc if bits else None)
    g, u = x.double().chunk(2, 1)
    value, _ = _parts(g, act)
    _near(y.t.view(rows, F), value * u, (6e-7 + 2e-7 * g.abs()) * (u * g).abs() + 1e-6 * (value * u).abs(), bf16)
    if bits:
        oc, osc = ref.quant_pack(to_np(x.view(-1)), mode=mode, bits=bits, block=block, frac_bits=fb, threads=4)
        np.testing.assert_array_equal(to_np(codes.t), oc)
        if blocked:
            np.testing.assert_array_equal(to_np(scales.t).view(np.uint32), osc.view(np.uint32))
        xhat = ref.dequant_unpack(oc, osc, n, mode=mode, bits=bits, block=block, frac_bits=fb, out_dtype=np.float32, threads=4)
        sf.gated_backward_dequant(codes.t, sc, act, mode, bits, block, fb, dy, dx.t.view(rows, 2 * F))
        g, u = torch.from_numpy(xhat).cuda().double().view(rows, 2 * F).chunk(2, 1)
        value, slope = _parts(g, act)
        d, got = dy.double(), dx.t.view(rows, 2 * F)
        rel = 6e-7 + 2e-7 * g.abs()
        _near(got[:, :F], d * u * slope, rel * (1 + g.abs()) * (d * u).abs() + 1e-6 * (d * u * slope).abs(), bf16)
        _near(got[:, F:], d * value, rel * (d * g).abs() + 1e-6 * (d * value).abs(), bf16)
    for b in (codes, scales, y, dx):
        b.check()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("act", [sf.ACT_SILU, sf.ACT_GELU])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,F,block", [(1, 32, 32), (3, 64, 64), (7, 96, 32), (5, 256, 256), (130, 384, 128), (1, 4096, 64), (33, 1408, 128)])
def test_block_caches(rows, F, block, bits, act, dtype):
    require_gpu()
    x, dy = _input(rows, F, DT[dtype], rows + F)
    _run(x, dy, act, sf.Q_BLOCK, bits, block, 0)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows,F", [(1, 8), (9, 24), (257, 40), (2, 2728)])
def test_fixed_point_caches_and_none(rows, F, dtype):
    """Widths that are no multiple of any block, with one factor for all and without a cache."""
    require_gpu()
    x, dy = _input(rows, F, DT[dtype], rows + F)
    for bits, fb in ((4, 1), (8, 4), (8, -2), (0, 0)):
        for act in (sf.ACT_SILU, sf.ACT_GELU):
            _run(x, dy, act, sf.Q_FIXED, bits, 0, fb)


def _off(got, want, tol, bf16):
    """The largest |got - want| beyond ``tol``, half a step of bf16 and the smallest numbers."""
    return float(((got.double() - want).abs() - tol - 1e-37 - (want.abs() * 2.0 ** -8 if bf16 else 0.0)).max())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("act", [sf.ACT_SILU, sf.ACT_GELU])
def test_gates_of_any_size(act, dtype):
    """Gates far from zero, where an activation is its gate or nothing and its slope one or zero: tolerances as the header states
    them, none of which grows with the size of a gate on the side where the result is nothing.  They count: for SiLU the
    argument's rounding and constant (7.3e-8 of |gate|), a step each of exp2 and the reciprocal, the sum's and two products' half
    steps; its slope's 1 - p keeps the absolute error of p, 1.8e-7, times the gate up to 17.4, beyond which 1 + e^-gate is 1; for
    GELU 2.1e-7 of erfc, 1.2e-7 of 2 - erfc and three half steps, and 4.1e-15 of a gate below -8.5."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(9)
    far = torch.logspace(0, 8, 2048, device="cuda")
    gate = torch.cat((torch.linspace(-40, 40, 8192, device="cuda"), torch.linspace(-6.0, -5.9, 512, device="cuda"),
                      torch.linspace(-105, -85, 512, device="cuda"), far, -far)).view(-1, 512)
    up = torch.randn(gate.shape, generator=g, device="cuda")
    x = torch.cat((gate, up), 1).to(DT[dtype])
    bf16 = dtype == "bf16"
    rows = gate.shape[0]
    y, codes, scales = torch.empty(rows, 512, dtype=x.dtype, device="cuda"), torch.empty(rows * 1024, dtype=torch.uint8, device="cuda"), torch.empty(rows * 32, device="cuda")
    sf.gated_quant_pack(x, act, sf.Q_BLOCK, 8, 32, 0, y, codes, scales)

    def tol(g, u, value):
        if act == sf.ACT_SILU:
            return (6e-7 + 1e-7 * g.abs()) * (value * u).abs() + 1e-36 * u.abs()
        return 4e-7 * g.abs().clamp(max=6.0) * u.abs() + 1e-6 * (value * u).abs() + 5e-15 * (g * u).abs()

    g64, u64 = x.double().chunk(2, 1)
    value, _ = _parts(g64, act)
    assert _off(y, value * u64, tol(g64, u64, value), bf16) <= 0
    dy = torch.randn(rows, 512, generator=g, device="cuda").to(x.dtype)
    dx = torch.empty_like(x)
    sf.gated_backward_dequant(codes, scales, act, sf.Q_BLOCK, 8, 32, 0, dy, dx)
    xhat = torch.empty(x.numel(), device="cuda")
    sf.dequant_unpack(codes, scales, sf.Q_BLOCK, 8, 32, 0, xhat)
    g64, u64 = xhat.double().view(rows, 1024).chunk(2, 1)
    value, slope = _parts(g64, act)
    d = dy.double()
    assert _off(dx[:, 512:], d * value, tol(g64, d, value), bf16) <= 0
    assert _off(dx[:, :512], d * u64 * slope, (6e-7 + 2e-7 * g64.abs().clamp(max=18.0)) * (d * u64).abs() + 1e-6 * (d * u64 * slope).abs(), bf16) <= 0


@pytest.mark.parametrize("dtype", DT)
def test_blocks_of_zeros_and_of_tiny_numbers_are_kept_as_zeros(dtype):
    require_gpu()
    x, dy = _input(4, 64, DT[dtype], 3)
    x[1] = 0.0
    x[2, 64:] = 1e-39
    _run(x, dy, sf.ACT_SILU, sf.Q_BLOCK, 8, 32, 0)


def test_the_backward_pass_is_the_slope_of_the_forward():
    """Differences of the forward pass in fp32, around values that the cache gives back exactly."""
    require_gpu()
    F, h = 64, 2.0 ** -9
    code = torch.arange(-64, 64, device="cuda").view(1, 2 * F).float() * 2.0 ** -5         # 8 bits, 5 of them of the fraction: exact
    ones = torch.ones(1, F, device="cuda")
    codes = torch.empty(2 * F, dtype=torch.uint8, device="cuda")
    for act in (sf.ACT_SILU, sf.ACT_GELU):
        def at(x):
            y = torch.empty(1, F, device="cuda")
            sf.gated_quant_pack(x, act, sf.Q_FIXED, 8, 0, 5, y, codes, None)
            return y.double()
        step = torch.zeros_like(code)
        step[:, :F] = h
        by_gate = (at(code + step) - at(code - step)) / (2 * h)
        by_up = (at(code + h - step) - at(code - h + step)) / (2 * h)
        at(code)
        dx = torch.empty(1, 2 * F, device="cuda")
        sf.gated_backward_dequant(codes, None, act, sf.Q_FIXED, 8, 0, 5, ones, dx)
        # |up| <= 2, the third derivative below 1: h^2 / 6 * 2 of the difference, 2 * 1e-6 * 4 / (2 h) of the roundings
        assert float((dx[:, :F] - by_gate).abs().max()) <= h * h / 3 + 4e-6 / h
        assert float((dx[:, F:] - by_up).abs().max()) <= 4e-6 / h


@pytest.mark.parametrize("bits,block", [(8, 64), (4, 32)])
def test_function(bits, block):
    require_gpu()
    x, dy = _input(6, 128, torch.float32, 5)
    x = x.view(2, 3, 256).requires_grad_(True)
    y = ag.GatedFunction.apply(x, sf.ACT_GELU, bits, block)
    assert y.shape == (2, 3, 128)
    (dx,) = torch.autograd.grad(y, x, dy.view(2, 3, 128).transpose(0, 1).contiguous().transpose(0, 1))
    want_y, codes = torch.empty(6, 128, device="cuda"), torch.empty(x.numel() * bits // 8, dtype=torch.uint8, device="cuda")
    scales, want = torch.empty(x.numel() // block, device="cuda"), torch.empty(6, 256, device="cuda")
    sf.gated_quant_pack(x.detach().view(6, 256), sf.ACT_GELU, sf.Q_BLOCK, bits, block, 0, want_y, codes, scales)
    sf.gated_backward_dequant(codes, scales, sf.ACT_GELU, sf.Q_BLOCK, bits, block, 0, dy, want)
    assert torch.equal(y.view(6, 128), want_y) and torch.equal(dx.view(6, 256), want)
    with torch.no_grad():
        assert torch.equal(ag.GatedFunction.apply(x, sf.ACT_GELU, bits, block), y)          # nothing kept, the same result


def test_arguments():
    require_gpu()
    x, y = torch.randn(4, 128, device="cuda"), torch.empty(4, 64, device="cuda")
    codes, scales = torch.empty(512, dtype=torch.uint8, device="cuda"), torch.empty(16, device="cuda")

    def status(*args, call=sf.gated_quant_pack):
        with pytest.raises(sf.SlimfitError) as e:
            call(*args)
        return e.value.status

    assert status(x, 2, sf.Q_BLOCK, 8, 32, 0, y, codes, scales) == sf.ERR_INVALID_ARG
    assert status(x, 0, sf.Q_BLOCK, 8, 128, 0, y, codes, scales) == sf.ERR_UNSUPPORTED       # a block would straddle the halves
    assert status(x, 0, sf.Q_BLOCK, 5, 32, 0, y, codes, scales) == sf.ERR_UNSUPPORTED
    assert status(codes, scales, 0, sf.Q_BLOCK, 0, 32, 0, y, x, call=sf.gated_backward_dequant) == sf.ERR_UNSUPPORTED
    both = torch.empty(4 * 192, device="cuda")
    assert status(both[:512].view(4, 128), 0, sf.Q_BLOCK, 0, 0, 0, both[256:512].view(4, 64), None, None) == sf.ERR_INVALID_ARG      # shared memory
    for bad in ((x, 0, sf.Q_BLOCK, 8, 32, 0, y, codes[:-1], scales), (x, 0, sf.Q_BLOCK, 8, 32, 0, y, codes, scales[:-1]),
                (x, 0, sf.Q_BLOCK, 8, 32, 0, y, None, None), (x, 0, sf.Q_BLOCK, 8, 32, 0, y.bfloat16(), codes, scales),
                (x[:, :127], 0, sf.Q_BLOCK, 8, 32, 0, y, codes, scales), (x.t().contiguous().t(), 0, sf.Q_BLOCK, 8, 32, 0, y, codes, scales),
                (x.cpu(), 0, sf.Q_BLOCK, 0, 32, 0, y, None, None), (x, 0, sf.Q_BLOCK, 0, 32, 0, y.cpu(), None, None)):
        with pytest.raises(ValueError):
            sf.gated_quant_pack(*bad)
    sf.gated_quant_pack(x[:0], 0, sf.Q_BLOCK, 8, 32, 0, y[:0], codes[:0], scales[:0])         # no rows


def test_more_rows_than_a_launch_takes():
    """2^30 vectors of y and some: two launches, the second's first row at the right place."""
    require_gpu()
    rows, F = (1 << 29) + 3, 16                                        # bf16: 2 vectors a row
    x = torch.zeros(rows, 2 * F, dtype=torch.bfloat16, device="cuda")
    x[-5:] = torch.randn(5, 2 * F, device="cuda").bfloat16()
    x[0] = x[-1]
    y = torch.empty(rows, F, dtype=torch.bfloat16, device="cuda")
    sf.gated_quant_pack(x, sf.ACT_SILU, sf.Q_BLOCK, 0, 0, 0, y, None, None)
    small = torch.empty(5, F, dtype=torch.bfloat16, device="cuda")
    sf.gated_quant_pack(x[-5:].clone(), sf.ACT_SILU, sf.Q_BLOCK, 0, 0, 0, small, None, None)
    assert torch.equal(y[-5:], small) and torch.equal(y[0], small[-1])
    assert int(torch.count_nonzero(y[1:-5])) == 0
