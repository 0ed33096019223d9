"""GPU: slimfit_heads_norm_rotate_forward / _backward against the formulas in 64 bits.  Tolerances count roundings: a value that
is a sum of terms is off by at most the stated number of fp32 half steps (2^-24) of the sum of their sizes, bf16 results by
half a step of bf16 (2^-8) more; codes and scales are those of quant_pack bit for bit, values are copies."""
import math

import pytest
import torch

from paper_2305_18513_amd import autograd as ag
from paper_2305_18513_amd import binding as sf
from tests.gpu_util import Guarded, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
H = 2.0 ** -24


class Case:
    """Inputs of both calls, on the GPU."""

    def __init__(self, B, T, Hq, Hk, D, R, dtype, pairing=sf.ROTARY_HALVES, norm=True, ids=False, bits=0, block=0, seed=0, eps=1e-6):
        g = torch.Generator(device="cuda").manual_seed(seed + 13 * T + D)
        self.B, self.T, self.Hq, self.Hk, self.D, self.R = B, T, Hq, Hk, D, R
        self.dtype, self.pairing, self.norm, self.bits, self.block, self.eps = dtype, pairing, norm, bits, block, eps

        def randn(*shape, dtype=dtype):
            return torch.randn(*shape, generator=g, device="cuda").to(dtype)

        self.qkv = randn(B, T, (Hq + 2 * Hk) * D, dtype=torch.float32)
        self.qkv.view(-1)[::37] *= 20.0
        self.qkv[0, 0, :D] = 0.0                                       # a head of zeros
        self.qkv = self.qkv.to(dtype)
        self.gq, self.gk = (randn(D, dtype=torch.float32) * 0.2 + 1 for _ in range(2)) if norm else (None, None)
        self.places = T + 50
        self.table = sf.rotary_table(self.places, R) if R else None
        self.ids = None
        if ids:
            self.ids = torch.randint(-3, self.places + 3, (B, T), generator=g, device="cuda").to(torch.int32)
            self.ids[0, 0] = self.places - 1
            self.ids[-1, -1] = -2147483648
        self.q_scale = 1 / math.sqrt(D)
        self.grads = randn(B, Hq, T, D), randn(B, Hk, D, T), randn(B, Hk, T, D)

    def angles(self):
        """(cos, sin) (B, T, 1, R / 2) in 64 bits, 1 and 0 where the place is outside of the table."""
        ids = torch.arange(self.T, device="cuda").expand(self.B, self.T) if self.ids is None else self.ids.long()
        inside = ((ids >= 0) & (ids < self.places))[..., None, None]
        row = self.table.double()[ids.clamp(0, self.places - 1)][:, :, None]
        return torch.where(inside, row[..., : self.R // 2], 1.0), torch.where(inside, row[..., self.R // 2 :], 0.0)

    def turn(self, y, back=False, size=False):
        """y turned; size: the sum of the sizes of the terms instead."""
        if not self.R:
            return y.abs() if size else y
        cos, sin = self.angles()
        sin = -sin if back else sin
        halves = self.pairing == sf.ROTARY_HALVES
        a, b = (y[..., : self.R // 2], y[..., self.R // 2 : self.R]) if halves else (y[..., 0 : self.R : 2], y[..., 1 : self.R : 2])
        if size:
            a, b, cos, sin, rest = a.abs(), b.abs(), cos.abs(), sin.abs(), y[..., self.R :].abs()
            first, second = a * cos + b * sin, b * cos + a * sin
        else:
            rest, first, second = y[..., self.R :], a * cos - b * sin, b * cos + a * sin
        first = torch.cat((first, second), -1) if halves else torch.stack((first, second), -1).flatten(-2)
        return torch.cat((first, rest), -1)

    def buffers(self):
        B, T, Hq, Hk, D = self.B, self.T, self.Hq, self.Hk, self.D
        n = B * T * (Hq + Hk) * D
        out = dict(q=Guarded(B * Hq * T * D, self.dtype), kt=Guarded(B * Hk * T * D, self.dtype), v=Guarded(B * Hk * T * D, self.dtype),
                   rstd=Guarded(B * T * (Hq + Hk) if self.norm else 0, torch.float32),
                   codes=Guarded(n * self.bits // 8, torch.uint8), scales=Guarded(n // self.block if self.bits else 0, torch.float32))
        return out

    def forward(self, out):
        B, T, Hq, Hk, D = self.B, self.T, self.Hq, self.Hk, self.D
        sf.heads_norm_rotate_forward(self.qkv, self.gq, self.gk, self.eps, self.table, self.pairing, self.ids, self.q_scale, self.bits, self.block,
                                     out["q"].t.view(B, Hq, T, D), out["kt"].t.view(B, Hk, D, T), out["v"].t.view(B, Hk, T, D),
                                     out["rstd"].t if self.norm else None, out["codes"].t if self.bits else None,
                                     out["scales"].t if self.bits else None)

    def backward(self, out, dqkv, dgq, dgk, workspace=None):
        reads = self.norm and not self.bits
        sf.heads_norm_rotate_backward(*self.grads, self.qkv if reads else None, out["codes"].t if self.bits else None,
                                      out["scales"].t if self.bits else None, self.bits, self.block, out["rstd"].t if self.norm else None,
                                      self.gq, self.gk, self.table, self.pairing, self.ids, self.q_scale, dqkv, dgq, dgk, workspace)


def _near(got, want, halves, size, bf16, what):
    tol = halves * H * size + (want.abs() * 2.0 ** -8 if bf16 else 0.0) + 1e-37
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), "%s: max excess %.3g of %.3g" % (what, float((off - tol).max()), float(want.abs().max()))


def _check(c):
    B, T, Hq, Hk, D = c.B, c.T, c.Hq, c.Hk, c.D
    bf16 = c.dtype == torch.bfloat16
    out = c.buffers()
    c.forward(out)
    torch.cuda.synchronize()
    for name, b in out.items():
        b.check()
    heads = c.qkv.view(B, T, Hq + 2 * Hk, D)
    assert torch.equal(out["v"].t.view(B, Hk, T, D), heads[:, :, Hq + Hk :].transpose(1, 2))
    x = heads[:, :, : Hq + Hk].double()
    y, rstd, gamma = x, 1.0, torch.ones((), device="cuda", dtype=torch.float64)
    if c.norm:
        # the sum of squares: E + log2(L) + 1 <= 16 roundings of positive terms, half of it in the root; its scaling, the addition and
        # the root itself (one step): 8 + 1 + 1 + 2
        rstd = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + c.eps)
        got = out["rstd"].t.view(B, T, Hq + Hk, 1).double()
        assert bool(((got - rstd).abs() <= 13 * H * rstd).all())
        gamma = torch.cat((c.gq.double().expand(Hq, D), c.gk.double().expand(Hk, D)))
        y = x * rstd * gamma
    # 13 of rstd, two products, the turn's two, the factor
    want, size = c.turn(y), c.turn(y, size=True)
    _near(out["q"].t.view(B, Hq, T, D), want[:, :, :Hq].transpose(1, 2) * c.q_scale, 19, size[:, :, :Hq].transpose(1, 2) * c.q_scale, bf16, "q")
    _near(out["kt"].t.view(B, Hk, D, T), want[:, :, Hq:].permute(0, 2, 3, 1), 19, size[:, :, Hq:].permute(0, 2, 3, 1), bf16, "kt")
    if c.bits:
        flat = heads[:, :, : Hq + Hk].contiguous().view(-1)
        codes, scales = torch.empty_like(out["codes"].t), torch.empty_like(out["scales"].t)
        sf.quant_pack(flat, sf.Q_BLOCK, c.bits, c.block, 0, codes, scales)
        assert torch.equal(out["codes"].t, codes) and torch.equal(out["scales"].t, scales)
        back = torch.empty(flat.numel(), device="cuda")
        sf.dequant_unpack(codes, scales, sf.Q_BLOCK, c.bits, c.block, 0, back)
        x = back.double().view(x.shape)

    dqkv, dgq, dgk = Guarded(c.qkv.numel(), c.dtype), Guarded(D, torch.float32), Guarded(D, torch.float32)
    c.backward(out, dqkv.t.view(c.qkv.shape), dgq.t if c.norm else None, dgk.t if c.norm else None)
    torch.cuda.synchronize()
    for b in (dqkv, dgq, dgk):
        b.check()
    got = dqkv.t.view(B, T, Hq + 2 * Hk, D)
    dq, dkt, dv = c.grads
    assert torch.equal(got[:, :, Hq + Hk :], dv.transpose(1, 2))
    d = torch.cat((dq.double().transpose(1, 2) * c.q_scale, dkt.double().permute(0, 3, 1, 2)), 2)
    g, g_size = c.turn(d, back=True), c.turn(d, back=True, size=True)
    if not c.norm:
        _near(got[:, :, : Hq + Hk], g, 4, g_size, bf16, "dqkv")
        return
    r = out["rstd"].t.view(B, T, Hq + Hk, 1).double()                  # the forward pass's: an input here
    xn = x * r
    by, by_size = g * xn, g_size * xn.abs()
    for name, h, to in (("dgamma_q", slice(0, Hq), dgq), ("dgamma_k", slice(Hq, None), dgk)):
        # a term: 3 of g, 2 of x~, its product; a lane's 32 terms, a workgroup's 64 lanes
        _near(to.t, by[:, :, h].sum((0, 1, 2)), 6 + 32 + 64, by_size[:, :, h].sum((0, 1, 2)), False, name)
    gy, gy_size = g * gamma, g_size * gamma.abs()
    dot, dot_size = (gy * xn).mean(-1, keepdim=True), (gy_size * xn.abs()).mean(-1, keepdim=True)
    # gy: 3 + 1; the mean: 4 + 2 of its terms, 16 of the sum, 1; the rest 3
    _near(got[:, :, : Hq + Hk], r * (gy - xn * dot), 30, r * (gy_size + xn.abs() * dot_size), bf16, "dqkv")


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("B,T,Hq,Hk,D,R,pairing,ids,bits,block", [
    (1, 1, 1, 1, 16, 16, 0, False, 0, 0), (1, 1, 4, 2, 64, 64, 0, True, 8, 64), (3, 1, 6, 3, 128, 128, 1, True, 8, 32),
    (2, 3, 2, 1, 32, 32, 0, True, 4, 32), (2, 5, 3, 3, 80, 48, 0, True, 0, 0), (1, 7, 8, 1, 96, 96, 1, False, 8, 32),
    (2, 65, 4, 2, 64, 32, 0, False, 4, 64), (1, 197, 3, 3, 64, 32, 1, True, 4, 32), (2, 64, 9, 3, 128, 128, 0, True, 8, 128),
    (1, 257, 2, 2, 256, 256, 0, False, 8, 256), (1, 72, 14, 2, 256, 64, 1, True, 8, 128), (5, 13, 2, 1, 8, 0, 0, False, 0, 0),
    (1, 1030, 2, 1, 16, 16, 0, True, 0, 0), (2, 520, 5, 1, 192, 192, 0, False, 4, 64), (70, 8, 2, 2, 40, 16, 1, True, 0, 0),
    (1, 128, 1, 1, 24, 16, 0, False, 0, 0), (1, 96, 12, 4, 112, 112, 0, True, 0, 0)])
def test_forward_and_backward(B, T, Hq, Hk, D, R, pairing, ids, bits, block, dtype):
    require_gpu()
    _check(Case(B, T, Hq, Hk, D, R, DT[dtype], pairing, True, ids, bits, block))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("pairing", [sf.ROTARY_HALVES, sf.ROTARY_ADJACENT])
@pytest.mark.parametrize("B,T,Hq,Hk,D,R", [(2, 33, 4, 2, 64, 64), (1, 64, 2, 2, 96, 32), (9, 1, 16, 4, 128, 128), (2, 40, 1, 1, 32, 0)])
def test_without_a_norm(B, T, Hq, Hk, D, R, pairing, dtype):
    require_gpu()
    _check(Case(B, T, Hq, Hk, D, R, DT[dtype], pairing, False, T % 2 == 1))


@pytest.mark.parametrize("dtype", DT)
def test_many_heads_and_rows(dtype):
    """Several heads a workgroup, several thousand partial sums."""
    require_gpu()
    _check(Case(16, 512, 32, 8, 128, 128, DT[dtype], bits=8, block=64))


def test_offsets_past_32_bits():
    """Rows past 2^31 elements and 4 GB of the projection: those at the end are what a call of them alone gives, to the bit."""
    require_gpu()
    T, few, Hq, Hk, D, bits, block = (1 << 21) + 37, 61, 6, 1, 128, 8, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    gains = [torch.rand(D, generator=g, device="cuda") + 0.5 for _ in range(2)]
    table = sf.rotary_table(100, D)

    def empty(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def both(qkv, dq, dkt, dv, ids):
        n = qkv.shape[1]
        q, kt, v, dqkv = empty(1, Hq, n, D), empty(1, Hk, D, n), empty(1, Hk, n, D), empty(*qkv.shape)
        rstd, codes, scales = empty(n, Hq + Hk, dtype=torch.float32), empty(n, (Hq + Hk) * D, dtype=torch.uint8), empty(n, (Hq + Hk) * D // block, dtype=torch.float32)
        sf.heads_norm_rotate_forward(qkv, *gains, 1e-6, table, sf.ROTARY_HALVES, ids, 0.125, bits, block, q, kt, v, rstd, codes.view(-1), scales)
        sf.heads_norm_rotate_backward(dq, dkt, dv, None, codes.view(-1), scales, bits, block, rstd, *gains, table, sf.ROTARY_HALVES, ids, 0.125, dqkv)
        return q[0].transpose(0, 1), kt[0].permute(2, 0, 1), v[0].transpose(0, 1), rstd, codes, scales, dqkv[0]

    qkv, dq, dkt, dv = empty(1, T, (Hq + 2 * Hk) * D).zero_(), empty(1, Hq, T, D).zero_(), empty(1, Hk, D, T).zero_(), empty(1, Hk, T, D).zero_()
    ids = torch.zeros(1, T, dtype=torch.int32, device="cuda")
    small = [torch.randn(*shape, generator=g, device="cuda").bfloat16() for shape in ((1, few, (Hq + 2 * Hk) * D), (1, Hq, few, D), (1, Hk, D, few), (1, Hk, few, D))]
    places = torch.randint(-2, 102, (1, few), generator=g, device="cuda").to(torch.int32)
    qkv[:, -few:], dq[:, :, -few:], dkt[..., -few:], dv[:, :, -few:], ids[:, -few:] = *small, places
    for far, near in zip(both(qkv, dq, dkt, dv, ids), both(*small, places)):
        assert torch.equal(far[-few:], near)
        assert not far[: T - few].any() if far.dtype != torch.float32 else bool((far[:100] == far[0]).all())


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D", [64, 80])
def test_rows_whose_squares_overflow(D, dtype):
    """The mean of the squares is infinite, rstd 0 and the row too, whether its lanes are all in the head or not."""
    require_gpu()
    c = Case(1, 9, 2, 1, D, 0, DT[dtype])
    c.qkv[0, 3] = 3e19
    out = c.buffers()
    c.forward(out)
    q = out["q"].t.view(1, 2, 9, D).float()
    assert bool(torch.isfinite(q).all()) and not q[:, :, 3].any() and bool(q[:, :, 2].any()) and not out["rstd"].t.view(9, 3)[3].any()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("pairing", [sf.ROTARY_HALVES, sf.ROTARY_ADJACENT])
@pytest.mark.parametrize("T", [1, 19])
def test_infinities_that_are_not_turned(T, pairing, dtype):
    """Without a norm, past the turned elements and in padding, every element is its own."""
    require_gpu()
    B, Hq, Hk, D, R = 3, 4, 2, 64, 32
    g = torch.Generator(device="cuda").manual_seed(5)
    heads = torch.randn(B, T, Hq + 2 * Hk, D, generator=g, device="cuda").to(DT[dtype])
    heads[:, :, :, R + 5 :: 7] = float("inf")
    ids = torch.zeros(B, T, dtype=torch.int32, device="cuda")
    ids[1], ids[2, ::2] = -1, 4                                                                    # padding
    heads[1, :, :, ::9] = float("-inf")
    heads[2, ::2, 1, 3] = float("inf")
    q, kt, v = (torch.empty(B, n, *rest, dtype=heads.dtype, device="cuda") for n, rest in ((Hq, (T, D)), (Hk, (D, T)), (Hk, (T, D))))
    back = torch.empty_like(heads).view(B, T, -1)
    for table, places in ((sf.rotary_table(4, R), ids), (None, None)):                             # place 0: the angles are 0
        x = heads.clone()
        if table is None:
            x[..., :R:3] = float("inf")
        sf.heads_norm_rotate_forward(x.view(B, T, -1), None, None, 0.0, table, pairing, places, 0.5, 0, 0, q, kt, v, None, None, None)
        assert torch.equal(q, x[:, :, :Hq].transpose(1, 2) * 0.5)
        assert torch.equal(kt, x[:, :, Hq : Hq + Hk].permute(0, 2, 3, 1)) and torch.equal(v, x[:, :, Hq + Hk :].transpose(1, 2))
        sf.heads_norm_rotate_backward(q, kt, v, None, None, None, 0, 0, None, None, None, table, pairing, places, 2.0, back)
        assert torch.equal(back.view_as(x), x)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("pairing", [sf.ROTARY_HALVES, sf.ROTARY_ADJACENT])
def test_infinities_that_are_not_turned_with_a_norm(pairing, dtype):
    """A row that holds an infinity has an rstd of 0: the element is NaN and the others are 0, past the turned ones and in padding, and
    an infinite gradient there is its own element's in the gains' sums."""
    require_gpu()
    c = Case(1, 21, 2, 1, 64, 32, DT[dtype], pairing)
    c.ids = torch.arange(21, dtype=torch.int32, device="cuda").view(1, 21)
    c.ids[0, 4] = -1
    heads = c.qkv.view(1, 21, 4, 64)
    heads[0, 0, 0, 0] = 1.0                                                     # (a head of zeros otherwise)
    heads[0, 4, :3, 3] = float("inf")                                           # in padding
    heads[0, 7, :3, 41] = float("-inf")                                         # past the turned elements
    out = c.buffers()
    c.forward(out)
    q, kt = out["q"].t.view(1, 2, 21, 64).float(), out["kt"].t.view(1, 1, 64, 21).float()
    for y in (q[0, 0], q[0, 1], kt[0, 0].t()):
        for row, at in ((4, 3), (7, 41)):
            assert bool(y[row, at].isnan()) and not y[row, :at].any() and not y[row, at + 1 :].any()
        assert bool(y[[0, 1, 2, 3, 5, 6, *range(8, 21)]].isfinite().all())
    c = Case(1, 21, 2, 1, 64, 32, DT[dtype], pairing)
    c.ids = torch.arange(21, dtype=torch.int32, device="cuda").view(1, 21)
    c.ids[0, 4] = -1
    out = c.buffers()
    c.forward(out)
    dq, dkt, _ = c.grads
    dq[0, 0, 4, 3], dq[0, 1, 7, 41] = float("inf"), float("inf")
    dkt[0, 0, 3, 4], dkt[0, 0, 41, 7] = float("inf"), float("inf")
    dqkv, dgq, dgk = torch.empty_like(c.qkv), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    c.backward(out, dqkv, dgq, dgk)
    for dg in (dgq, dgk):
        assert [i for i, fine in enumerate(dg.isfinite().tolist()) if not fine] == [3, 41]


def test_plain_splits_are_split_heads():
    """Neither norm nor rotation, keys not shared: what split_heads and merge_heads do, to the bit."""
    require_gpu()
    for dtype in DT.values():
        c = Case(2, 70, 3, 3, 64, 0, dtype, norm=False)
        c.q_scale = 0.125
        out = c.buffers()
        c.forward(out)
        q, kt, v = (torch.empty(2, 3, *s, dtype=dtype, device="cuda") for s in ((70, 64), (64, 70), (70, 64)))
        sf.split_heads(c.qkv, 0.125, q, kt, v)
        assert torch.equal(out["q"].t, q.view(-1)) and torch.equal(out["kt"].t, kt.view(-1)) and torch.equal(out["v"].t, v.view(-1))
        dqkv, want = torch.empty_like(c.qkv), torch.empty_like(c.qkv)
        c.backward(out, dqkv, None, None)
        sf.merge_heads(*c.grads, 0.125, want)
        assert torch.equal(dqkv, want)


def test_frozen_norms_and_results_that_repeat():
    require_gpu()
    c = Case(4, 130, 8, 2, 64, 64, torch.bfloat16, bits=8, block=64)
    out = c.buffers()
    c.forward(out)
    first, again = torch.empty_like(c.qkv), torch.empty_like(c.qkv)
    dg = [torch.empty(64, device="cuda") for _ in range(4)]
    need = sf.heads_norm_rotate_workspace(torch.bfloat16, 4, 130, 8, 2, 64)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")           # NaN
    c.backward(out, first, dg[0], dg[1], ws)
    c.backward(out, again, dg[2], dg[3])
    assert torch.equal(first, again) and torch.equal(dg[0], dg[2]) and torch.equal(dg[1], dg[3]) and bool(torch.isfinite(dg[0]).all())
    again.fill_(7)
    c.backward(out, again, None, None)                                          # frozen
    assert torch.equal(first, again)
    with pytest.raises(sf.SlimfitError) as e:
        c.backward(out, again, dg[2], dg[3], ws[:-16])
    assert e.value.status == sf.ERR_WORKSPACE


def test_no_tokens():
    require_gpu()
    dg = [torch.full((64,), 5.0, device="cuda") for _ in range(2)]
    e = lambda *s: torch.empty(*s, device="cuda")                               # noqa: E731
    sf.heads_norm_rotate_forward(e(2, 0, 256), e(64), e(64), 1e-6, None, 0, None, 1.0, 0, 0, e(2, 2, 0, 64), e(2, 1, 64, 0), e(2, 1, 0, 64),
                                 e(0), None, None)
    sf.heads_norm_rotate_backward(e(2, 2, 0, 64), e(2, 1, 64, 0), e(2, 1, 0, 64), e(2, 0, 256), None, None, 0, 0, e(0), e(64), e(64), None, 0, None, 1.0,
                                  e(2, 0, 256), dg[0], dg[1])
    assert not dg[0].any() and not dg[1].any()                                  # sums of nothing


@pytest.mark.parametrize("frozen", [False, True])
@pytest.mark.parametrize("bits", [0, 8])
def test_function(bits, frozen):
    """The autograd wrapper's gradients are the calls', with gradients in any layout."""
    require_gpu()
    c = Case(2, 48, 4, 2, 64, 64, torch.float32, ids=True, bits=bits, block=64 if bits else 0)
    x = c.qkv.clone().requires_grad_(True)
    gq, gk = (g.clone().requires_grad_(not frozen) for g in (c.gq, c.gk))
    outs = ag.HeadsNormRotateFunction.apply(x, gq, gk, 4, 2, c.table, c.pairing, c.ids, c.q_scale, c.eps, bits, 64)
    out = c.buffers()
    c.forward(out)
    for o, name in zip(outs, ("q", "kt", "v")):
        assert torch.equal(o.reshape(-1), out[name].t)
    leaves = [x] if frozen else [x, gq, gk]
    grads = torch.autograd.grad(outs, leaves, [g.transpose(2, 3).contiguous().transpose(2, 3) for g in c.grads])
    dqkv, dgq, dgk = torch.empty_like(c.qkv), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    c.backward(out, dqkv, dgq, dgk)
    for got, want in zip(grads, (dqkv, dgq, dgk)):
        assert torch.equal(got, want)
    # one output alone used: the others' gradients count as zeros
    outs = ag.HeadsNormRotateFunction.apply(x, gq, gk, 4, 2, c.table, c.pairing, c.ids, c.q_scale, c.eps, bits, 64)
    (dx,) = torch.autograd.grad(outs[0], x, c.grads[0])
    assert bool(torch.isfinite(dx).all()) and not dx[..., 4 * 64 :].any() and bool(dx[..., : 4 * 64].any())


def test_arguments():
    require_gpu()
    c = Case(2, 8, 4, 2, 64, 64, torch.float32, bits=8, block=32)
    e = lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda")      # noqa: E731
    good = dict(qkv=c.qkv, gamma_q=c.gq, gamma_k=c.gk, eps=1e-6, table=c.table, pairing=0, position_ids=None, q_scale=1.0, bits=8, block=32,
                q=e(2, 4, 8, 64), kt=e(2, 2, 64, 8), v=e(2, 2, 8, 64), rstd=e(16 * 6), codes=e(16 * 6 * 64, dtype=torch.uint8), scales=e(16 * 6 * 2))
    sf.heads_norm_rotate_forward(**good)
    for name, value, status in (("block", 48, sf.ERR_UNSUPPORTED), ("block", 128, sf.ERR_UNSUPPORTED), ("bits", 3, sf.ERR_UNSUPPORTED),
                                ("pairing", 2, sf.ERR_INVALID_ARG), ("eps", -1.0, sf.ERR_INVALID_ARG), ("eps", float("nan"), sf.ERR_INVALID_ARG),
                                ("table", e(7, 64), sf.ERR_INVALID_ARG), ("table", e(50, 20), sf.ERR_UNSUPPORTED), ("table", e(50, 72), sf.ERR_INVALID_ARG),
                                ("v", good["kt"].view(2, 2, 8, 64), sf.ERR_INVALID_ARG)):
        with pytest.raises(sf.SlimfitError) as err:
            sf.heads_norm_rotate_forward(**dict(good, **{name: value}))
        assert err.value.status == status, name
    for name, value in (("q", e(2, 4, 8, 32)), ("kt", e(2, 2, 8, 64)), ("v", e(2, 1, 8, 64)), ("rstd", None), ("rstd", e(95)), ("gamma_k", None),
                        ("gamma_q", e(63)), ("gamma_q", e(64, dtype=torch.bfloat16)), ("position_ids", torch.zeros(2, 8, device="cuda")),
                        ("position_ids", torch.zeros(15, dtype=torch.int32, device="cuda")), ("codes", good["codes"][:-1]), ("scales", None),
                        ("qkv", c.qkv.bfloat16()), ("qkv", c.qkv.transpose(0, 1)), ("table", c.table.double()), ("table", c.table.cpu())):
        with pytest.raises(ValueError):
            sf.heads_norm_rotate_forward(**dict(good, **{name: value}))
    odd = dict(good, qkv=e(2, 8, 8 * 36), q=e(2, 4, 8, 36), kt=e(2, 2, 36, 8), v=e(2, 2, 8, 36), gamma_q=e(36), gamma_k=e(36), table=None, bits=0)
    sf.heads_norm_rotate_forward(**odd)
    for t in ("qkv", "q", "kt", "v"):
        odd[t] = odd[t].bfloat16()
    with pytest.raises(sf.SlimfitError) as err:
        sf.heads_norm_rotate_forward(**odd)                                     # 72 bytes a head
    assert err.value.status == sf.ERR_UNSUPPORTED
