"""GPU: slimfit_weight_grad_dequant against the product in 64 bits, at the tolerances the header states."""
import pytest
import torch

from paper_2305_18513_amd import autograd as ag
from paper_2305_18513_amd import binding as sf
from tests.gpu_util import Guarded, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _cached(M, K, bits, block, seed, dtype=torch.float32):
    """(codes, scales, x^ in 64 bits) of an M x K input."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, generator=g, device="cuda")
    x.view(-1)[::31] *= 20.0
    x = x.to(dtype)
    codes = torch.empty(sf.packed_bytes(M * K, bits), dtype=torch.uint8, device="cuda")
    scales = torch.empty(sf.num_blocks(M * K, block), device="cuda")
    sf.quant_pack(x.view(-1), sf.Q_BLOCK, bits, block, 0, codes, scales)
    code = torch.empty(M * K, device="cuda")
    sf.dequant_unpack(codes, torch.ones_like(scales), sf.Q_BLOCK, bits, block, 0, code)
    return codes, scales, (code.double().view(-1, block) * scales.double()[:, None]).view(M, K)


def _check(got, dy, x):
    M = dy.shape[0]
    want, total = dy.double().t() @ x, dy.double().abs().t() @ x.abs()
    if got.dtype == torch.bfloat16:
        tol = (2.0 ** -8 + (2 * M + 8) * 2.0 ** -23) * total + 2.0 ** -8 * want.abs()
    else:
        tol = (2 * M + 8) * 2.0 ** -23 * total
    off = (got.double() - want).abs()
    assert bool((off <= tol + M * 2.0 ** -120).all()), "max excess %.3g" % float((off - tol).max())
    # and, roundings being independent, an error of the size of their root of sum of squares: 2^-8 / sqrt 3 of an entry and of the result
    # where they are bf16's, a few steps of fp32 otherwise
    if M > 0 and float(want.norm()) > 0:
        assert float(off.norm() / want.norm()) <= (2.0 ** -8 * 1.2 if got.dtype == torch.bfloat16 else 2e-6 * max(1.0, float(total.norm() / want.norm()) ** 0.5))


def _run(M, N, K, bits, block, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 7)
    codes, scales, x = _cached(M, K, bits, block, seed, dtype)
    dy = (torch.randn(M, N, generator=g, device="cuda") * 0.1).to(dtype)
    dw = Guarded(N * K, dtype)
    sf.weight_grad_dequant(dy, codes, scales, bits, block, dw.t.view(N, K))
    torch.cuda.synchronize()
    dw.check()
    _check(dw.t.view(N, K), dy, x)
    return dy, codes, scales, dw.t.view(N, K)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K,block", [(1, 2, 32, 32), (1, 128, 256, 256), (63, 8, 64, 64), (64, 127, 160, 32), (65, 1, 128, 128), (200, 129, 192, 64),
                                         (31, 1003, 96, 32), (129, 256, 128, 64), (777, 130, 768, 256)])
def test_sizes(M, N, K, block, bits, dtype):
    require_gpu()
    _run(M, N, K, bits, block, DT[dtype], M + N)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("M,N,K,block", [(4100, 129, 160, 32), (2049, 64, 128, 64), (9001, 256, 384, 128), (5000, 770, 768, 64)])
def test_long_sums_are_shared_out(M, N, K, block, dtype):
    require_gpu()
    assert sf.weight_grad_dequant_workspace(DT[dtype], block, M, N, K) > 0
    dy, codes, scales, dw = _run(M, N, K, 8, block, DT[dtype], M)
    again = torch.empty_like(dw)
    need = sf.weight_grad_dequant_workspace(DT[dtype], block, M, N, K)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")           # NaN: everything that is read was written
    sf.weight_grad_dequant(dy, codes, scales, 8, block, again, ws)
    assert torch.equal(again, dw)
    with pytest.raises(sf.SlimfitError) as e:
        sf.weight_grad_dequant(dy, codes, scales, 8, block, again, ws[:-16])
    assert e.value.status == sf.ERR_WORKSPACE


# bf16 sizes whose tiles are 256 x 128 (test_weight_plan_cpu.py checks that they are): rows of dw and columns that end inside a tile,
# several bands and columns of tiles, sums in one part and in several
WIDE = [(333, 1032, 5280), (130, 2312, 2208), (70, 4104, 1312), (4100, 2312, 416), (6000, 520, 5280)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K", WIDE)
def test_wide_tiles(M, N, K, bits):
    require_gpu()
    assert (sf.weight_grad_dequant_workspace(torch.bfloat16, 32, M, N, K) > 0) == (M > 4000)
    dy, codes, scales, dw = _run(M, N, K, bits, 32, torch.bfloat16, M)
    again = torch.empty_like(dw)
    sf.weight_grad_dequant(dy, codes, scales, bits, 32, again)
    assert torch.equal(again, dw)


@pytest.mark.parametrize("dtype", DT)
def test_no_rows_and_zeros(dtype):
    require_gpu()
    dw = torch.full((40, 64), 3.0, dtype=DT[dtype], device="cuda")
    sf.weight_grad_dequant(torch.empty(0, 40, dtype=DT[dtype], device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda"),
                           torch.empty(0, device="cuda"), 8, 32, dw)
    assert int(torch.count_nonzero(dw)) == 0
    # blocks of zeros (scale 0) and the lowest code, -128 and -8
    for bits in (8, 4):
        codes = torch.full((64 * 64 * bits // 8,), 0x80 if bits == 8 else 0x88, dtype=torch.uint8, device="cuda")
        scales = torch.ones(64 * 2, device="cuda")
        scales[::3] = 0.0
        dy = torch.ones(64, 40, dtype=DT[dtype], device="cuda")
        sf.weight_grad_dequant(dy, codes, scales, bits, 32, dw)
        want = (scales.view(64, 2).double().sum(0) * -(128 if bits == 8 else 8)).repeat_interleave(32).expand(40, 64)
        assert torch.equal(dw.double(), want.to(DT[dtype]).double())


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e18, 1e30])
def test_fp32_entries_of_any_size(size):
    require_gpu()
    codes, scales, x = _cached(100, 128, 8, 64, 3)
    dy = torch.randn(100, 64, device="cuda") * size
    dw = torch.empty(64, 128, device="cuda")
    sf.weight_grad_dequant(dy, codes, scales, 8, 64, dw)
    _check(dw, dy, x)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("bits", [8, 4])
def test_inputs_of_the_largest_size(bits, dtype):
    """Inputs of the type's lowest and largest value: times zero gradients, of masked rows, they are nothing, times small ones finite."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(70, 64, generator=g, device="cuda").to(DT[dtype])
    x[3], x[40, ::2] = torch.finfo(x.dtype).min, torch.finfo(x.dtype).max
    dy = torch.randn(70, 24, generator=g, device="cuda").to(DT[dtype])
    dy[3], dy[40] = 0.0, 0.0
    codes, scales = torch.empty(70 * 64 * bits // 8, dtype=torch.uint8, device="cuda"), torch.empty(70 * 2, device="cuda")
    sf.quant_pack(x.view(-1), sf.Q_BLOCK, bits, 32, 0, codes, scales)
    code = torch.empty(70 * 64, device="cuda")
    sf.dequant_unpack(codes, torch.ones_like(scales), sf.Q_BLOCK, bits, 32, 0, code)
    x_hat = (code.double().view(-1, 32) * scales.double()[:, None]).view(70, 64)
    dw = torch.empty(24, 64, dtype=x.dtype, device="cuda")
    for rows in (dy, torch.where(torch.arange(70, device="cuda")[:, None] == 3, 2.0 ** -40, 0.0).expand(70, 24).to(x.dtype).contiguous()):
        sf.weight_grad_dequant(rows, codes, scales, bits, 32, dw)
        assert bool(dw.isfinite().all())
        _check(dw, rows, x_hat)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("M,N,K,block", [(100, 40, 128, 64), (131, 41, 96, 32), (70, 3, 64, 32), (4200, 24, 64, 32)])
def test_fp32_gradients_that_are_not_finite_or_overflow_with_the_scale(M, N, K, block, bits):
    """Infinities and NaN come out where the product has them, and gradients that are infinite once the scale is on them, or once
    rounded to a bf16 part, are finite where their codes make them so."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(M)
    codes, scales, x = _cached(M, K, bits, block, M)
    dy = torch.randn(M, N, generator=g, device="cuda") * 0.1
    code = torch.randint(-7, 8, (M, K), generator=g, device="cuda")
    large = 3.4e38                                                       # a step of bf16 below 2^128 and a quarter: rounds to infinity
    code[11] = code[11].sign()
    code[13] = 0
    scales.view(M, -1)[11] = 1.0
    scales.view(M, -1)[13] = 4.0
    dy[11, 0] = large
    dy[13, 1] = 2e38                                                     # times the scale: past fp32
    dy[M - 1, N - 1] = float("-inf")
    dy[M - 1, N - 2] = float("nan") if N > 3 else 0.0
    if N > 3:
        dy[2, 2], dy[9, 3], dy[M // 2, 3] = float("inf"), float("inf"), float("-inf")
    raw = code.to(torch.int8).view(torch.uint8).view(-1)
    codes.copy_(raw if bits == 8 else (raw[0::2] & 15) | (raw[1::2] << 4))
    x = (code.double().view(-1, block) * scales.double().view(-1)[:, None]).view(M, K)
    dw = Guarded(N * K, torch.float32)
    sf.weight_grad_dequant(dy, codes, scales, bits, block, dw.t.view(N, K))
    dw.check()
    got = dw.t.view(N, K).double()
    want, total = (sum((a[i : i + 50, :, None] * b[i : i + 50, None]).sum(0) for i in range(0, M, 50)) for a, b in ((dy.double(), x), (dy.double().abs(), x.abs())))
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
    assert bool((got == want)[want.isinf()].all()) and bool(want[:2].isfinite().all()) and bool(want.isinf().any())
    fine = want.isfinite()
    assert bool(((got - want).abs() <= (2 * M + 8) * 2.0 ** -23 * total + M * 2.0 ** -120)[fine].all())


def test_offsets_past_32_bits():
    """Rows whose codes, and whose gradients, lie past 4 GB."""
    require_gpu()
    K, M = 4096, (1 << 20) + 5                                           # codes of 4.3 GB
    codes = torch.zeros(M * K, dtype=torch.uint8, device="cuda")
    codes.view(M, K)[-70:] = torch.randint(0, 256, (70, K), device="cuda", dtype=torch.int32).to(torch.uint8)
    scales = torch.full((M * K // 256,), 0.01, device="cuda")
    dy = torch.randn(M, 2, device="cuda").bfloat16()
    dw, want = (torch.empty(2, K, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sf.weight_grad_dequant(dy, codes, scales, 8, 256, dw)
    x = codes.view(M, K)[-70:].view(torch.int8).double() * 0.009999999776482582
    _check(dw, dy[-70:], x)
    dy = torch.zeros((1 << 20) + 65, 4096, dtype=torch.bfloat16, device="cuda")                    # 8.6 GB
    dy[-65:] = torch.randn(65, 4096, device="cuda").bfloat16()
    codes, scales, x = _cached(dy.shape[0], 32, 8, 32, 5, torch.bfloat16)
    dw = torch.empty(4096, 32, dtype=torch.bfloat16, device="cuda")
    sf.weight_grad_dequant(dy, codes, scales, 8, 32, dw)
    _check(dw, dy[-65:], x[-65:])


@pytest.mark.parametrize("dtype", DT)
def test_linear_function(dtype):
    """An active layer whose weight gradient comes straight from the codes, and what stays with the other route."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(3)
    for K, block in ((256, 64), (96, 64)):                                                         # 96: blocks straddle rows
        x = torch.randn(4, 50, K, generator=g, device="cuda").to(DT[dtype]).requires_grad_(True)
        w = (torch.randn(136, K, generator=g, device="cuda") * 0.05).to(DT[dtype]).requires_grad_(True)
        b = torch.randn(136, generator=g, device="cuda").to(DT[dtype]).requires_grad_(True)
        dy = torch.randn(4, 50, 136, generator=g, device="cuda").to(DT[dtype])
        calls, kept = [], sf.weight_grad_dequant
        ag.sf.weight_grad_dequant = lambda *a: (calls.append(1), kept(*a))[1]
        try:
            outs = [ag.LinearFunction.apply(x, w, b, 8, block, straight) for straight in (False, True)]
            grads = [torch.autograd.grad(o, (x, w, b), dy) for o in outs]
        finally:
            ag.sf.weight_grad_dequant = kept
        assert len(calls) == (K == 256)
        assert torch.equal(outs[0], outs[1]) and torch.equal(grads[0][0], grads[1][0]) and torch.equal(grads[0][2], grads[1][2])
        # the same x^ (bf16: rounded alike) in sums of another order: a rounding of the result each, and the sums' own
        scale = dy.double().abs().view(-1, 136).t() @ x.detach().double().abs().view(-1, K)
        tol = 2 * 2.0 ** -8 * grads[0][1].double().abs() + 1e-4 * scale if dtype == "bf16" else 4 * 200 * 2.0 ** -23 * scale
        assert bool(((grads[0][1].double() - grads[1][1].double()).abs() <= tol).all())


def test_linear_function_past_what_a_call_takes():
    """A layer of more outputs than that: torch's product, as without ``straight``."""
    require_gpu()
    N, K = (1 << 20) + 8, 64
    x, w = torch.randn(3, K, device="cuda"), torch.randn(N, K, device="cuda").requires_grad_(True)
    dy = torch.randn(3, N, device="cuda")
    grads = [torch.autograd.grad(ag.LinearFunction.apply(x, w, None, 8, 64, straight), w, dy)[0] for straight in (False, True)]
    assert torch.equal(*grads)


def test_arguments():
    require_gpu()
    codes, scales, _ = _cached(64, 96, 8, 32, 0)
    dy, dw = torch.randn(64, 40, device="cuda"), torch.empty(40, 96, device="cuda")

    def status(*args):
        with pytest.raises(sf.SlimfitError) as e:
            sf.weight_grad_dequant(*args)
        return e.value.status

    assert status(dy, codes, scales, 8, 64, dw) == sf.ERR_UNSUPPORTED                              # a block would straddle two rows
    assert status(dy, codes, scales, 8, 48, dw) == sf.ERR_UNSUPPORTED
    assert status(dy, codes, scales, 6, 32, dw) == sf.ERR_UNSUPPORTED
    for bad in ((dy, codes[:-1], scales, 8, 32, dw), (dy, codes, scales[:-1], 8, 32, dw), (dy, codes, scales, 8, 32, dw.bfloat16()),
                (dy[:, :39], codes, scales, 8, 32, dw), (dy, codes, scales, 8, 32, dw[:39]), (dy.t().contiguous().t(), codes, scales, 8, 32, dw),
                (dy.cpu(), codes, scales, 8, 32, dw), (dy, codes.cpu(), scales, 8, 32, dw)):
        with pytest.raises(ValueError):
            sf.weight_grad_dequant(*bad)
