"""Attention's forward and backward pass and its position bias on the GPU against the formulas in 64 bits, element by element, within
bounds that follow from the number of roundings on each way."""
import math

import pytest
import torch

from paper_2305_18513_amd import binding as sf
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                             # a rounding to fp32
UB = 2.0 ** -8                                             # to bf16


def inputs(B, Tq, Tk, Hq, Hk, D, dtype, layout, seed=0, columns=False, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") * spread).to(dtype)  # noqa: E731
    if layout == sf.HEADS_APART:
        return rand(B, Hq, Tq, D), rand(B, Hk, D, Tk), rand(B, Hk, Tk, D), rand(B, Tq, Hq, D)
    if columns:                                            # columns of rows that hold more
        rq, rk = rand(B, Tq, Hq + 3, D), rand(B, Tk, 2 * Hk + 1, D)
        return rq[:, :, 1 : Hq + 1], rk[:, :, :Hk], rk[:, :, Hk + 1 :], rand(B, Tq, Hq, D)
    return rand(B, Tq, Hq, D), rand(B, Tk, Hk, D), rand(B, Tk, Hk, D), rand(B, Tq, Hq, D)


def rows_of(t, layout, keys=False):
    """(B, heads, tokens, D) in 64 bits."""
    if layout == sf.HEADS_APART:
        return t.double().transpose(2, 3) if keys else t.double()
    return t.double().transpose(1, 2)


class Reference:
    def __init__(self, q, k, v, do, layout, scale, causal, lengths, table, bucket_of):
        self.low = q.dtype == torch.bfloat16
        q, k, v = rows_of(q, layout), rows_of(k, layout, True), rows_of(v, layout)
        B, Hq, Tq, D = q.shape
        Hk, Tk = k.shape[1:3]
        self.group, self.sizes = Hq // Hk, (B, Tq, Tk, Hq, Hk, D)
        if lengths is not None:                            # what is past a sequence's end is not looked at
            gone = (torch.arange(Tk, device="cuda")[None] >= lengths[:, None])[:, None, :, None]
            k, v = k.masked_fill(gone, 0.0), v.masked_fill(gone, 0.0)
        self.q, self.scale = q, scale
        self.k, self.v = k.repeat_interleave(self.group, 1), v.repeat_interleave(self.group, 1)
        i, j = torch.arange(Tq, device="cuda")[:, None], torch.arange(Tk, device="cuda")[None]
        s = q @ self.k.transpose(2, 3) * scale
        self.size = q.abs() @ self.k.abs().transpose(2, 3) * scale                # of s's terms
        self.at = None
        if table is not None:
            self.buckets = table.shape[0]
            self.at = bucket_of.long()[j - i + Tq - 1]
            inside = (self.at >= 0) & (self.at < self.buckets)
            bias = torch.where(inside[None], table.double().t()[:, self.at.clamp(0, self.buckets - 1)], 0.0)
            s = s + bias
            self.size = self.size + torch.where(torch.isinf(bias), 0.0, bias.abs())
            self.at = torch.where(inside, self.at, -1)
        seen = torch.ones(B, 1, Tq, Tk, dtype=torch.bool, device="cuda")
        if causal:
            seen = seen & (j - i <= Tk - Tq)
        if lengths is not None:
            seen = seen & (j < lengths[:, None, None, None])
        s = s.masked_fill(~seen, -math.inf)
        self.top = s.amax(-1, keepdim=True) if Tk else s.new_full((B, Hq, Tq, 1), -math.inf)
        some = self.top > -math.inf
        e = torch.exp(s - torch.where(some, self.top, 0.0))
        self.total = e.sum(-1, keepdim=True)
        self.p = torch.where(some, e / torch.where(some, self.total, 1.0), 0.0)
        self.out = self.p @ self.v
        # a p's relative error: s's (D products and sums, scale, bias) in it and in the maximum, the exponent's own roundings (a
        # difference, a product, the constant's half step), the exponential's 2, the sum over the keys, the division.  l's has all of that too.
        live = s > -math.inf
        off = torch.where(live, self.size, 0.0) * (D + 6) * U + torch.where(live, s - self.top, 0.0).abs() * 4 * U
        off = off + torch.where(some, self.top, 0.0).abs().clamp(max=1e4) * 4 * U + 4 * U
        worst = off.amax(-1, keepdim=True) if Tk else off.new_zeros(B, Hq, Tq, 1)
        self.p_off = 2 * (off + worst) + (Tk + 8) * U
        self.top_off = worst
        self.total_off = 2 * worst + (Tk + 4) * U
        if do is not None:
            self.backward(do.double().transpose(1, 2))

    def rounded(self, off, value):
        """With the result's own rounding, and what lies below the type's normal numbers."""
        return off * (1 + UB) + UB * value.abs() + 2.0 ** -120 if self.low else off + U * value.abs() + 2.0 ** -120

    def product_off(self):
        return UB if self.low else 0.0                     # of an operand that is rounded before a product

    def out_off(self):
        Tk = self.sizes[2]
        return ((self.p_off + self.product_off() + (Tk + 4) * U) * self.p) @ self.v.abs()

    def backward(self, do):
        B, Tq, Tk, Hq, Hk, D = self.sizes
        part = self.product_off()
        dp, size = do @ self.v.transpose(2, 3), do.abs() @ self.v.abs().transpose(2, 3)
        delta = (do * self.out).sum(-1, keepdim=True)
        o_off = self.rounded(self.out_off(), self.out)
        delta_off = (do.abs() * (o_off + (D + 2) * U * self.out.abs())).sum(-1, keepdim=True)
        ds = self.p * (dp - delta)
        ds_off = self.p_off * ds.abs() + self.p * (1 + self.p_off) * ((D + 2) * U * size + delta_off + 2 * U * (dp.abs() + delta.abs())) + 2 * U * ds.abs()
        self.ds, used = ds, ds_off + part * (ds.abs() + ds_off)
        self.dq, dq_off = ds @ self.k * self.scale, (used + (Tk + 4) * U * ds.abs()) @ self.k.abs() * self.scale
        n = Tq * self.group
        share = lambda t: t.view(B, Hk, self.group, Tk, D).sum(2)  # noqa: E731
        self.dk = share(ds.transpose(2, 3) @ self.q) * self.scale
        dk_off = share((used + (n + 4) * U * ds.abs()).transpose(2, 3) @ self.q.abs()) * self.scale
        self.dv = share(self.p.transpose(2, 3) @ do)
        dv_off = share((self.p * (self.p_off + part + (n + 4) * U)).transpose(2, 3) @ do.abs())
        self.offs = dict(dq=self.rounded(dq_off, self.dq), dk=self.rounded(dk_off, self.dk), dv=self.rounded(dv_off, self.dv))
        if self.at is not None:
            add = lambda t: torch.stack([(t * (self.at == b)).sum((0, 2, 3)) for b in range(self.buckets)])  # noqa: E731
            self.dtable = add(ds)
            self.offs["dtable"] = self.rounded(add(ds_off + 40 * U * ds.abs()), self.dtable)


def within(got, want, off, what):
    bad = (got - want).abs() > off
    assert not bool(bad.any()) and not bool(torch.isnan(got).any()), "%s: %d of %d, worst %.3g of its bound" % (
        what, int(bad.sum()), bad.numel(), float(((got - want).abs() / off).max()))


class Call:
    """One forward and backward pass with outputs between sentinels (77), as columns of wider rows where the operands are."""

    def __init__(self, q, k, v, do, layout, scale, causal=False, lengths=None, table=None, bucket_of=None, columns=False):
        self.args = (q, k, v, layout, scale, causal, lengths, table, bucket_of)
        self.do, self.kept = do, []
        self.out = self.new(do.shape, q.dtype)
        B, Tq, Hq, D = do.shape
        self.stats = self.new((B, Hq, Tq, 2), torch.float32)
        if columns:
            B, Tk, Hk, D = k.shape
            self.wide_q, self.wide_k = (torch.full(s, 77.0, dtype=q.dtype, device="cuda") for s in ((B, Tq, Hq + 3, D), (B, Tk, 2 * Hk + 1, D)))
            self.dq, self.dk, self.dv = self.wide_q[:, :, 1 : Hq + 1], self.wide_k[:, :, :Hk], self.wide_k[:, :, Hk + 1 :]
        else:
            self.dq, self.dk, self.dv = (self.new(t.shape, t.dtype) for t in (q, k, v))
        self.dtable = None if table is None else self.new(table.shape, table.dtype)
        self.columns = columns

    def new(self, shape, dtype):
        n = math.prod(shape)
        raw = torch.full((n + 64,), 77.0, dtype=dtype, device="cuda")
        self.kept.append((raw, n))
        return raw[32 : 32 + n].view(shape) if n else torch.empty(shape, dtype=dtype, device="cuda")

    def forward(self, **more):
        sf.attention_forward(*self.args, self.out, self.stats, **more)
        return self

    def backward(self, **more):
        sf.attention_backward(self.do, *self.args, self.out, self.stats, self.dq, self.dk, self.dv, self.dtable, **more)
        return self

    def outputs(self):
        return [t for t in (self.out, self.stats, self.dq, self.dk, self.dv, self.dtable) if t is not None]

    def check(self):
        q, k, v, layout, scale, causal, lengths, table, bucket_of = self.args
        r = Reference(q, k, v, self.do, layout, scale, causal, lengths, table, bucket_of)
        out = rows_of(self.out, sf.HEADS_ROWS)
        within(out, r.out, r.rounded(r.out_off(), r.out), "out")
        top, total = self.stats[..., :1].double(), self.stats[..., 1:].double()
        none = r.top == -math.inf
        assert torch.equal(top == -math.inf, none) and bool((total[none] == 0).all()) and bool((out[none.expand_as(out)] == 0).all())
        within(torch.where(none, 0.0, top), torch.where(none, 0.0, r.top), r.top_off + U * torch.where(none, 0.0, r.top).abs(), "maximum")
        within(total, r.total, r.total_off * r.total + 1e-40, "sum")
        within(rows_of(self.dq, layout), r.dq, r.offs["dq"], "dq")
        within(rows_of(self.dk, layout, True), r.dk, r.offs["dk"], "dk")
        within(rows_of(self.dv, layout), r.dv, r.offs["dv"], "dv")
        if self.dtable is not None:
            within(self.dtable.double(), r.dtable, r.offs["dtable"], "dtable")
        for raw, n in self.kept:
            assert bool((raw[:32] == 77).all()) and bool((raw[32 + n :] == 77).all())
        if self.columns:
            Hq, Hk = q.shape[2], k.shape[2]
            assert bool((self.wide_q[:, :, [0, Hq + 1, Hq + 2]] == 77).all()) and bool((self.wide_k[:, :, Hk] == 77).all())
        return r


SHAPES = [(1, 1, 1, 1, 1, 8), (2, 1, 70, 4, 2, 64), (2, 33, 65, 4, 1, 40), (1, 128, 128, 2, 2, 32), (3, 129, 257, 6, 3, 80), (2, 64, 200, 3, 3, 96),
          (1, 300, 300, 2, 1, 128), (2, 200, 77, 2, 2, 64), (5, 7, 3, 2, 1, 16), (1, 31, 513, 7, 1, 128), (2, 197, 197, 2, 2, 64)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("layout,columns", [(sf.HEADS_ROWS, False), (sf.HEADS_ROWS, True), (sf.HEADS_APART, False)], ids=["rows", "columns", "apart"])
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
def test_against_64_bits(shape, dtype, causal, layout, columns, bias):
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    q, k, v, do = inputs(*shape, dtype, layout, seed=Tq + Tk, columns=columns)
    lengths = torch.tensor([(0, Tk + 9, Tk // 2, 1, -3)[b % 5] for b in range(B)], dtype=torch.int32, device="cuda") if columns or bias else None
    table = of = None
    if bias:
        table = torch.randn(9, Hq, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
        of = sf.distance_buckets(Tq, Tk, 9, 40, both_ways=not causal)
    Call(q, k, v, do, layout, D ** -0.5, causal, lengths, table, of, columns).forward().backward().check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_odd_head_sizes(dtype):
    require_gpu()
    for D in ((4, 12, 36, 68, 100, 124) if dtype == torch.float32 else (8, 24, 56, 72, 104, 120)):
        q, k, v, do = inputs(2, 70, 90, 2, 1, D, dtype, sf.HEADS_ROWS, seed=D)
        Call(q, k, v, do, sf.HEADS_ROWS, 0.3, True).forward().backward().check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_large_logits(dtype):
    require_gpu()
    q, k, v, do = inputs(2, 100, 130, 2, 2, 64, dtype, sf.HEADS_ROWS, seed=4, spread=3.0)
    Call(q, k, v, do, sf.HEADS_ROWS, 0.5).forward().backward().check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", [sf.HEADS_ROWS, sf.HEADS_APART])
def test_what_is_past_the_lengths_is_not_looked_at(dtype, layout):
    require_gpu()
    shape = (3, 50, 150, 4, 2, 64)
    q, k, v, do = inputs(*shape, dtype, layout, seed=2)
    lengths = torch.tensor([70, 0, 128], dtype=torch.int32, device="cuda")
    table, of = torch.randn(5, 4, device="cuda").to(dtype), sf.distance_buckets(50, 150, 5, 30)
    clean = Call(q, k, v, do, layout, 0.2, False, lengths, table, of).forward().backward()
    clean.check()
    k, v = k.clone(), v.clone()
    for b, n in enumerate(lengths.tolist()):
        for bad, at in ((float("nan"), n), (float("inf"), n + 7), (-float("inf"), n + 1)):
            if layout == sf.HEADS_ROWS:
                k[b, at:, :, ::3] = bad
                v[b, at:] = bad
            else:
                k[b, :, ::3, at:] = bad
                v[b, :, at:] = bad
    spoilt = Call(q, k, v, do, layout, 0.2, False, lengths, table, of).forward().backward()
    assert all(torch.equal(a, b) for a, b in zip(clean.outputs(), spoilt.outputs()))
    past = torch.arange(150, device="cuda")[None] >= lengths[:, None]
    dk = rows_of(spoilt.dk, layout, True).transpose(1, 2)
    dv = rows_of(spoilt.dv, layout).transpose(1, 2)
    assert bool((dk[past] == 0).all()) and bool((dv[past] == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["infinite", "lowest", "all infinite", "all lowest", "outside"])
def test_biases_that_mask(dtype, kind):
    """-infinity takes pairs out, as a mask does; the type's lowest value counts where a query has nothing else, and the buckets
    outside of the table add nothing."""
    require_gpu()
    Tq, Tk = 100, 140
    q, k, v, do = inputs(2, Tq, Tk, 2, 2, 32, dtype, sf.HEADS_ROWS, seed=3)
    table = torch.randn(4, 2, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda").to(dtype)
    low = -math.inf if "infinite" in kind else torch.finfo(dtype).min
    of = sf.distance_buckets(Tq, Tk, 4, 20)
    if kind == "outside":
        of[::3] = -1
        of[1::7] = 4
        of[2::11] = 2 ** 31 - 1
    elif kind.startswith("all"):
        table[:, 0] = low                                  # the first head sees nothing, or everything alike
    else:
        table[1] = low
    call = Call(q, k, v, do, sf.HEADS_ROWS, 0.2, True, None, table, of).forward().backward()
    r = call.check()
    if kind == "all lowest":                               # a query's keys count alike: logits below half a step of the lowest value vanish
        assert float((call.stats[:, 0, :, 1].double() - torch.arange(Tk - Tq + 1, Tk + 1, device="cuda")).abs().max()) == 0.0
    if kind == "all infinite":
        assert bool((call.out[:, :, 0] == 0).all()) and bool((call.dq[:, :, 0] == 0).all()) and bool((r.total[:, 0] == 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_first_keys_that_are_not_seen(dtype):
    """Some queries of a wave see nothing of the first tiles, and what they see later is 1000 lower than what their neighbours saw."""
    require_gpu()
    Tq, Tk = 64, 320
    q, k, v, do = inputs(1, Tq, Tk, 2, 2, 64, dtype, sf.HEADS_ROWS, seed=12)
    table = torch.tensor([[0.0, 2.0], [-math.inf, -math.inf], [-1000.0, -900.0]], device="cuda").to(dtype)
    far = torch.arange(1 - Tq, Tk, device="cuda")
    of = torch.where(far >= 200, 2, torch.where(far >= -20, 1, 0)).to(torch.int32)
    call = Call(q, k, v, do, sf.HEADS_ROWS, 0.125, False, None, table, of).forward().backward()
    r = call.check()
    assert bool((r.top[0, 0, :20] < -900).all()) and bool((r.top[0, 0, 21:] > -10).all())


def test_no_keys_no_queries_no_batch():
    require_gpu()
    for dtype in (torch.float32, torch.bfloat16):
        for B, Tq, Tk in ((2, 5, 0), (2, 0, 5), (0, 5, 5)):
            for layout in (sf.HEADS_ROWS, sf.HEADS_APART):
                q, k, v, do = inputs(B, Tq, Tk, 4, 2, 16, dtype, layout)
                table, of = torch.randn(3, 4, device="cuda").to(dtype), torch.zeros(max(0, Tq + Tk - 1), dtype=torch.int32, device="cuda")
                c = Call(q, k, v, do, layout, 0.5, True, None, table, of).forward().backward()
                torch.cuda.synchronize()
                assert all(bool((t == 0).all()) for t in (c.out, c.dq, c.dk, c.dv, c.dtable))
                assert bool((c.stats[..., 0] == -math.inf).all()) and bool((c.stats[..., 1] == 0).all())


def test_the_same_call_gives_the_same_bits_on_any_stream():
    require_gpu()
    for dtype in (torch.float32, torch.bfloat16):
        q, k, v, do = inputs(3, 300, 280, 6, 2, 64, dtype, sf.HEADS_APART, seed=5)
        table, of = torch.randn(12, 6, device="cuda").to(dtype), sf.distance_buckets(300, 280, 12, 60)
        lengths = torch.tensor([280, 100, 7], dtype=torch.int32, device="cuda")
        calls = [Call(q, k, v, do, sf.HEADS_APART, 0.125, False, lengths, table, of) for _ in range(3)]
        torch.cuda.synchronize()
        calls[0].forward().backward()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        need = [sf.attention_workspace(dtype, sf.HEADS_APART, 3, 300, 280, 6, 2, 64, True, back) for back in (False, True)]
        held = [[torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in need] for _ in range(2)]      # NaN, wherever it is read
        torch.cuda.synchronize()
        for c, s, ws in zip(calls[1:], streams, held):     # side by side
            c.forward(workspace=ws[0], stream=s.cuda_stream)
        for c, s, ws in zip(calls[1:], streams, held):
            c.backward(workspace=ws[1], stream=s.cuda_stream)
        torch.cuda.synchronize()
        for c in calls[1:]:
            assert all(torch.equal(a, b) for a, b in zip(calls[0].outputs(), c.outputs()))
        with pytest.raises(ValueError):                    # whose workspace would be freed too early
            calls[0].backward(stream=streams[0].cuda_stream)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_captured_and_replayed(dtype):
    require_gpu()
    shape = (2, 150, 170, 4, 2, 64)
    table, of = torch.randn(12, 4, device="cuda").to(dtype), sf.distance_buckets(150, 170, 12, 60)
    lengths = torch.tensor([170, 90], dtype=torch.int32, device="cuda")
    q, k, v, do = inputs(*shape, dtype, sf.HEADS_APART, seed=0)
    c = Call(q, k, v, do, sf.HEADS_APART, 0.125, True, lengths, table, of)
    e = Call(q, k, v, do, sf.HEADS_APART, 0.125, True, lengths, table, of)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward().backward()
    for seed in (1, 2, 3):
        for to, now in zip((q, k, v, do), inputs(*shape, dtype, sf.HEADS_APART, seed=seed)):
            to.copy_(now)
        lengths.copy_(torch.tensor([170 - seed, 40 * seed], dtype=torch.int32))
        table.mul_(0.9)
        e.forward().backward()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(c.outputs(), e.outputs()))
    c.check()


def test_gradients_against_differences():
    """Along a random direction the loss <out, dout> of the kernel's own forward pass changes as the gradients say.  A central difference
    of step h is off by h^2 / 6 of the third derivative (its terms are of the loss's size times the direction's to the third: with
    h = 1/16 below 2e-3 of them) and by the loss's own rounding over h: 2^-24 times 16 times the square root of its terms."""
    require_gpu()
    q, k, v, do = inputs(2, 40, 60, 4, 2, 32, torch.float32, sf.HEADS_ROWS, seed=6)
    g = torch.Generator(device="cuda").manual_seed(7)
    table, of = torch.randn(6, 4, generator=g, device="cuda"), sf.distance_buckets(40, 60, 6, 20)
    base = Call(q, k, v, do, sf.HEADS_ROWS, 32 ** -0.5, False, None, table, of).forward().backward()
    h = 1.0 / 16
    for name, at, grad in (("q", q, base.dq), ("k", k, base.dk), ("v", v, base.dv), ("table", table, base.dtable)):
        way = torch.randn(at.shape, generator=g, device="cuda")
        way /= way.norm()

        def loss(sign):
            new = {n: t + sign * h * way if n == name else t for n, t in (("q", q), ("k", k), ("v", v), ("table", table))}
            c = Call(new["q"], new["k"], new["v"], do, sf.HEADS_ROWS, 32 ** -0.5, False, None, new["table"], of).forward()
            return (c.out.double() * do.double()).sum()

        got, want = float((loss(1) - loss(-1)) / (2 * h)), float((grad.double() * way.double()).sum())
        size = float(grad.double().norm())                 # a unit direction's change is at most that
        assert abs(got - want) <= 2e-3 * size + 16 * U * math.sqrt(do.numel()), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 1, 2100, 8, 2, 128), (70, 1, 1500, 8, 8, 64), (3, 5, 1030, 14, 2, 96), (2, 32, 700, 4, 4, 32), (1, 1, 5000, 7, 1, 80), (300, 2, 300, 2, 2, 40),
                                   (600, 1, 700, 1, 1, 128), (2, 30, 900, 6, 2, 128)], ids=lambda s: "x".join(map(str, s)))
def test_few_queries(shape, dtype):
    """Single tokens and a few over long keys, which are shared out over workgroups, some of several tiles, with sequences of any length."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    g = torch.Generator(device="cuda").manual_seed(B)
    lengths = torch.randint(0, Tk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lengths[0] = Tk
    for causal, bias, layout in ((False, False, sf.HEADS_ROWS), (True, True, sf.HEADS_ROWS), (True, False, sf.HEADS_APART)):
        q, k, v, do = inputs(*shape, dtype, layout, seed=Tk, columns=layout == sf.HEADS_ROWS)
        table = torch.randn(9, Hq, generator=g, device="cuda").to(dtype) if bias else None
        of = sf.distance_buckets(Tq, Tk, 9, 400, False) if bias else None
        c = Call(q, k, v, do, layout, D ** -0.5, causal, lengths if not causal or bias else None, table, of).forward()
        r = Reference(q, k, v, None, layout, D ** -0.5, *c.args[5:])
        out = rows_of(c.out, sf.HEADS_ROWS)
        within(out, r.out, r.rounded(r.out_off(), r.out), "out")
        none = r.top == -math.inf
        top, total = c.stats[..., :1].double(), c.stats[..., 1:].double()
        assert torch.equal(top == -math.inf, none) and bool((total[none] == 0).all()) and bool((out[none.expand_as(out)] == 0).all())
        within(torch.where(none, 0.0, top), torch.where(none, 0.0, r.top), r.top_off + U * torch.where(none, 0.0, r.top).abs(), "maximum")
        within(total, r.total, r.total_off * r.total + 1e-40, "sum")
        for raw, n in c.kept:
            assert bool((raw[:32] == 77).all()) and bool((raw[32 + n :] == 77).all())


def test_offsets_past_32_bits():
    """Keys and values as columns of rows so long that the last lie past 2^32 elements."""
    require_gpu()
    row, Tk, D = 1 << 20, 4200, 64
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of GPU memory")
    wide, dwide = (torch.empty(1, Tk, row // D, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, k, v, do = inputs(1, 70, Tk, 2, 2, D, torch.bfloat16, sf.HEADS_ROWS, seed=9)
    wide[:, :, 5:7], wide[:, :, -2:] = k, v
    a = Call(q, k, v, do, sf.HEADS_ROWS, 0.125).forward().backward()
    b = Call(q, wide[:, :, 5:7], wide[:, :, -2:], do, sf.HEADS_ROWS, 0.125)
    b.dk, b.dv = dwide[:, :, 3:5], dwide[:, :, -2:]
    b.forward().backward()
    assert all(torch.equal(x, y) for x, y in zip(a.outputs(), b.outputs()))
    a.check()


def test_many_tokens():
    require_gpu()
    for dtype, T in ((torch.bfloat16, 4097), (torch.float32, 2500)):
        q, k, v, do = inputs(1, T, T, 2, 1, 64, dtype, sf.HEADS_APART, seed=T)
        table, of = torch.randn(32, 2, device="cuda").to(dtype), sf.distance_buckets(T, T, 32, 500, False)
        Call(q, k, v, do, sf.HEADS_APART, 0.125, True, None, table, of).forward().backward().check()


class RightDelta(Reference):
    """Bounds without the rounding of out in them.  With e the most that delta from a rounded out may be off, ds is first formed with it,
    p (dp - delta) + e p, and rounded so for a product; the sum of a row's ds then gives e back, but for 32 bits' roundings, and e times
    sum of p k, of which p is rounded to bf16, is taken off.  Where the right delta is there from the start it is less than that."""

    def backward(self, do):
        super().backward(do)
        B, Tq, Tk, Hq, Hk, D = self.sizes
        dp, size = do @ self.v.transpose(2, 3), do.abs() @ self.v.abs().transpose(2, 3)
        delta = (do * self.out).sum(-1, keepdim=True)
        e = (do.abs() * (self.rounded(self.out_off(), self.out) + (D + 2) * U * self.out.abs())).sum(-1, keepdim=True)
        first = self.ds.abs() + e * self.p
        # a ds's 32 bits: p's own, dp's D products and sums, the difference; delta's: all of its row's, their sum, and delta' times what the p are off from 1
        one = self.p_off * first + self.p * (1 + self.p_off) * ((D + 2) * U * size + 2 * U * (dp.abs() + delta.abs() + e)) + 2 * U * first
        delta_off = (one + (Tk + 8) * U * first + self.p * self.p_off * (delta.abs() + e)).sum(-1, keepdim=True)
        ds_off = one + self.p * delta_off
        n, group = Tq * self.group, self.group
        share = lambda t: t.view(B, Hk, group, Tk, D).sum(2)  # noqa: E731
        dq_off = (ds_off + UB * (first + e * self.p) * (1 + UB) + (Tk + 4) * U * (first + e * self.p)) @ self.k.abs() * self.scale
        dk_off = share((ds_off + UB * (self.ds.abs() + ds_off) + (n + 4) * U * self.ds.abs()).transpose(2, 3) @ self.q.abs()) * self.scale
        self.offs["dq"], self.offs["dk"] = self.rounded(dq_off, self.dq), self.rounded(dk_off, self.dk)
        if self.at is not None:
            add = lambda t: torch.stack([(t * (self.at == b)).sum((0, 2, 3)) for b in range(self.buckets)])  # noqa: E731
            self.offs["dtable"] = self.rounded(add(ds_off + 40 * U * self.ds.abs()), self.dtable)


@pytest.mark.parametrize("T,D,buckets", [(7, 128, 0), (128, 128, 0), (128, 104, 0), (100, 128, 2), (300, 64, 0), (300, 96, 0), (300, 40, 0), (300, 64, 2), (260, 96, 2),
                                         (1, 128, 0), (1, 64, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_where_few_keys_take_all(T, D, buckets, causal):
    """A rounded out's part in delta stays out of dq and dk (heads past 96: up to 128 keys), and out of a bucket that all keys share, whose sum is 0."""
    require_gpu()
    q, k, v, do = inputs(2, T, T, 4, 2, D, torch.bfloat16, sf.HEADS_ROWS, seed=T + D, spread=1.5)
    table, of = None, None
    if buckets:
        table = torch.randn(buckets, 4, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
        of = torch.zeros(2 * T - 1, dtype=torch.int32, device="cuda")
    call = Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, None, table, of)
    call.forward()
    call.backward()
    ref = RightDelta(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, None, table, of)
    within(rows_of(call.dq, sf.HEADS_ROWS), ref.dq, ref.offs["dq"], "dq")
    within(rows_of(call.dk, sf.HEADS_ROWS, True), ref.dk, ref.offs["dk"], "dk")
    if buckets:
        within(call.dtable.double(), ref.dtable, ref.offs["dtable"], "dtable")


@pytest.mark.parametrize("shape", [(35, 129, 140, 2, 1, 32), (11, 150, 300, 6, 3, 64), (17, 197, 197, 4, 4, 84), (34, 130, 200, 2, 2, 128)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
def test_fp32_of_many_workgroups(shape, causal, bias):
    """Where keys are not shared out: more workgroups of 128 queries than half of the card's units."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    assert B * Hq * ((Tq + 127) // 128) > 128
    q, k, v, do = inputs(*shape, torch.float32, sf.HEADS_ROWS, seed=Tk)
    lengths = torch.tensor([(Tk, 0, Tk // 2, 1, Tk + 9)[b % 5] for b in range(B)], dtype=torch.int32, device="cuda") if bias else None
    table = of = None
    if bias:
        table = torch.randn(9, Hq, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
        of = sf.distance_buckets(Tq, Tk, 9, 40, both_ways=not causal)
    Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, lengths, table, of).forward().backward().check()


@pytest.mark.parametrize("shape", [(1, 1, 700, 2, 1, 32), (1, 700, 700, 1, 1, 64), (2, 513, 1100, 3, 1, 96), (1, 1031, 530, 2, 2, 128), (3, 640, 64, 1, 1, 40), (1, 1500, 1500, 1, 1, 128),
                                   (1, 40, 2100, 4, 4, 64)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("kind", ["all", "causal_lengths", "bias", "causal_bias_lengths", "apart"])
def test_blocks_whose_tiles_are_shared_out(shape, dtype, kind):
    """So few blocks that workgroups share their tiles out, also more workgroups than a block has tiles (early queries, short sequences)."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    layout, causal = sf.HEADS_APART if kind == "apart" else sf.HEADS_ROWS, "causal" in kind
    q, k, v, do = inputs(*shape, dtype, layout, seed=Tq, columns=kind == "bias")
    lengths = torch.tensor([(Tk - 5, 0, 70)[b % 3] for b in range(B)], dtype=torch.int32, device="cuda") if "lengths" in kind else None
    table = of = None
    if "bias" in kind:
        table = torch.randn(9, Hq, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
        of = sf.distance_buckets(Tq, Tk, 9, 400, both_ways=not causal)
    Call(q, k, v, do, layout, D ** -0.5, causal, lengths, table, of, kind == "bias").forward().backward().check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 4500, 140, 5, 1, 32), (1, 140, 9000, 2, 2, 64), (40, 700, 600, 4, 1, 64), (30, 130, 1100, 6, 1, 128)], ids=lambda s: "x".join(map(str, s)))
def test_blocks_of_one_side_are_shared_out(shape, dtype):
    """Tiles shared out for the queries' sums alone, or for the keys'."""
    require_gpu()
    q, k, v, do = inputs(*shape, dtype, sf.HEADS_ROWS, seed=shape[1])
    Call(q, k, v, do, sf.HEADS_ROWS, shape[5] ** -0.5, True).forward().backward().check()


@pytest.mark.parametrize("T,D", [(300, 128), (601, 104), (1100, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_wide_heads_where_one_key_takes_most(T, D, causal):
    """Logits far apart: delta is formed anew for 32 queries where one key takes more than half of some query; the others' dq is looked at elsewhere."""
    require_gpu()
    q, k, v, do = inputs(2, T, T, 4 if T < 1000 else 16, 2, D, torch.bfloat16, sf.HEADS_ROWS, seed=T + D, spread=1.7)
    call = Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal).forward().backward()
    ref = RightDelta(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, None, None, None)
    whole = T // 32 * 32
    most = call.stats[:, :, :whole, 1].reshape(*call.stats.shape[:2], -1, 32)
    anew = (most < 2).any(-1).repeat_interleave(32, -1)[..., None]
    assert float(anew.float().mean()) > 0.25
    off = torch.where(anew, ref.offs["dq"][:, :, :whole], math.inf)
    within(rows_of(call.dq, sf.HEADS_ROWS)[:, :, :whole], ref.dq[:, :, :whole], off, "dq")
    within(rows_of(call.dk, sf.HEADS_ROWS, True), ref.dk, ref.offs["dk"], "dk")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_most_buckets(dtype):
    """1024 of them, each with a distance or two of its own, over tiles that are shared out."""
    require_gpu()
    q, k, v, do = inputs(1, 700, 650, 2, 1, 32, dtype, sf.HEADS_ROWS, seed=11)
    table = torch.randn(1024, 2, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dtype)
    of = (torch.arange(700 + 650 - 1, dtype=torch.int32, device="cuda") * 7) % 1100          # some outside of the table
    Call(q, k, v, do, sf.HEADS_ROWS, 0.2, False, None, table, of).forward().backward().check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
def test_shared_out_tiles_captured_and_replayed(dtype, bias):
    """The shares' sums meet in one order: eager, captured and replayed calls give the same bits, also after other operands went through the graph."""
    require_gpu()
    q, k, v, do = inputs(1, 900, 1100, 2, 1, 128, dtype, sf.HEADS_ROWS, seed=2)
    table = torch.randn(9, 2, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype) if bias else None
    of = sf.distance_buckets(900, 1100, 9, 400, both_ways=False) if bias else None
    c = Call(q, k, v, do, sf.HEADS_ROWS, 0.1, True, None, table, of).forward().backward()
    want = [t.clone() for t in c.outputs()]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        c.forward().backward()
        with torch.cuda.graph(graph, stream=stream):
            c.forward().backward()
    torch.cuda.current_stream().wait_stream(stream)
    kept = q.clone()
    for turn in range(3):
        for t in c.outputs():
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(c.outputs(), want)), turn
        q.copy_(q.flip(0).roll(1, 1))
        graph.replay()
        assert not torch.equal(c.out, want[0])
        q.copy_(kept)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 16, 40, 200])
def test_the_last_tokens_over_all_keys_are_the_whole_passes_last_rows(dtype, n):
    """A decoder with a position bias that varies, trained over whole rows and asked for a few tokens over the keys before them."""
    require_gpu()
    T, Hq, Hk, D = 700, 4, 2, 64
    q, k, v, do = inputs(2, T, T, Hq, Hk, D, dtype, sf.HEADS_ROWS, seed=T + n)
    table = (2.0 * torch.randn(32, Hq, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")).to(dtype)
    whole = Reference(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, True, None, table, sf.distance_buckets(T, T, 32, 128, both_ways=False))
    few = Call(q[:, -n:].contiguous(), k, v, do[:, -n:].contiguous(), sf.HEADS_ROWS, D ** -0.5, True, None, table, sf.distance_buckets(n, T, 32, 128, both_ways=False))
    few.forward().backward()
    within(rows_of(few.out, sf.HEADS_ROWS), whole.out[:, :, -n:], whole.rounded(whole.out_off(), whole.out)[:, :, -n:], "out")
    within(rows_of(few.dq, sf.HEADS_ROWS), whole.dq[:, :, -n:], whole.offs["dq"][:, :, -n:], "dq")
    few.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 70, 150, 4, 2, 64), (40, 150, 150, 4, 2, 64), (40, 130, 260, 4, 2, 128), (1, 1, 700, 4, 2, 96)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_a_nan_that_is_seen_is_in_all_that_it_is_in_by_the_formulas(shape, dtype, bias, what):
    """In a query, a key or a value of one head: NaN in each result that it enters and in no other, and other sequences' results are those without it."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    group = Hq // Hk
    q, k, v, do = inputs(*shape, dtype, sf.HEADS_ROWS, seed=Tk)
    table = torch.randn(9, Hq, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype) if bias else None
    of = sf.distance_buckets(Tq, Tk, 9, 40) if bias else None
    clean = Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, False, None, table, of).forward().backward()
    at = dict(q=q.clone(), k=k.clone(), v=v.clone())
    at[what][B - 1, (Tq if what == "q" else Tk) // 2, (Hq if what == "q" else Hk) - 1, 3] = math.nan      # of the last sequence, in the last head
    got = Call(at["q"], at["k"], at["v"], do, sf.HEADS_ROWS, D ** -0.5, False, None, table, of).forward().backward()
    q, k, v, do = (t[-1].double().transpose(0, 1) for t in (at["q"], at["k"].repeat_interleave(group, 2), at["v"].repeat_interleave(group, 2), do))
    p = torch.softmax(q @ k.mT, -1)                        # (NaN wherever the scaled and biased ones are)
    out = p @ v
    ds = p * (do @ v.mT - (do * out).sum(-1, keepdim=True))
    shared = lambda t: t.view(Hk, group, Tk, D).sum(1)  # noqa: E731
    for name, t in dict(out=out, dq=ds @ k, dk=shared(ds.mT @ q), dv=shared(p.mT @ do)).items():
        nan, new, old = torch.isnan(t).transpose(0, 1), getattr(got, name), getattr(clean, name)
        assert bool(nan.any()) == (what != "v" or name != "dv"), name
        assert torch.equal(torch.isnan(new[-1]), nan) and torch.equal(new[:-1], old[:-1]), name
    if bias:
        i, j = torch.arange(Tq, device="cuda")[:, None], torch.arange(Tk, device="cuda")[None]
        bucket = of.long()[j - i + Tq - 1]
        assert torch.equal(torch.isnan(got.dtable), torch.stack([(torch.isnan(ds) & (bucket == b)).any(2).any(1) for b in range(9)]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-37, 1e-38, 2.0 ** -126, 2.0 ** -149, 1.7e38, 3e38], ids=str)
@pytest.mark.parametrize("shape", [(36, 200, 200, 4, 2, 64), (36, 130, 150, 4, 2, 128), (1, 3, 700, 4, 2, 32)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
def test_the_least_and_the_largest_scales(dtype, scale, shape, bias):
    """Logits of all but 0, whose keys count alike (or by their bias); from 2^127 on, where scale log2 e has no number, the call is refused."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    q, k, v, do = inputs(*shape, dtype, sf.HEADS_ROWS, seed=Tk)
    if scale > 1:
        q.zero_()
    table = torch.randn(9, Hq, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype) if bias else None
    of = sf.distance_buckets(Tq, Tk, 9, 40, both_ways=False) if bias else None
    call = Call(q, k, v, do, sf.HEADS_ROWS, scale, True, None, table, of)
    if scale >= 2.0 ** 127:
        for one in (call.forward, call.backward):
            with pytest.raises(sf.SlimfitError):
                one()
        return
    call.forward().backward()
    r = Reference(q, k, v, do, sf.HEADS_ROWS, float(torch.tensor(scale, dtype=torch.float32)), True, None, table, of)
    assert torch.equal(call.stats[..., 1] > 0, r.total[..., 0] > 0)
    within(rows_of(call.out, sf.HEADS_ROWS), r.out, r.rounded(r.out_off(), r.out), "out")
    within(call.stats[..., 1:].double(), r.total, r.total_off * r.total + 1e-40, "sum")
    within(rows_of(call.dv, sf.HEADS_ROWS), r.dv, r.offs["dv"], "dv")
    if bias:
        within(call.dtable.double(), r.dtable, r.offs["dtable"], "dtable")
    if scale < 1:
        within(rows_of(call.dq, sf.HEADS_ROWS), r.dq, r.offs["dq"], "dq")
        within(rows_of(call.dk, sf.HEADS_ROWS, True), r.dk, r.offs["dk"], "dk")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(41, 1500, 1400, 50, 25, 32), (1, 9000, 9100, 32, 32, 32), (700, 130, 1100, 12, 12, 32)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
def test_sums_by_distance_in_turns(shape, dtype, causal):
    """More sums than are held: blocks of queries in turns (five, five and two of twelve; 64 and seven; one and one), each added to the sums of those
    before, also where a replayed graph finds another call's sums there."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    q, k, v, do = inputs(*shape, dtype, sf.HEADS_ROWS, seed=Tk)
    lengths = torch.tensor([(Tk, 0, Tk // 2, 1, Tk + 9)[b % 5] for b in range(B)], dtype=torch.int32, device="cuda")
    table = torch.randn(9, Hq, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    of = sf.distance_buckets(Tq, Tk, 9, 200, both_ways=not causal)
    call = Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, lengths, table, of).forward().backward()
    want = [t.clone() for t in call.outputs()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.backward()
    for _ in range(2):
        for t in (call.dq, call.dk, call.dv, call.dtable):
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(call.outputs(), want))
    del graph, want
    per, heads = max(1, 20_000_000 // (Hq * Tq * Tk)), 2 if B == 1 else Hq                # what is looked at in 64 bits at a time
    dtable, off = torch.zeros(2, 9, Hq, dtype=torch.float64, device="cuda")
    for b in range(0, B, per):
        for h in range(0, Hq, heads):
            few, q_heads, k_heads = slice(b, b + per), slice(h, h + heads), slice(h, h + heads) if B == 1 else slice(0, Hk)
            r = Reference(q[few, :, q_heads], k[few, :, k_heads], v[few, :, k_heads], do[few, :, q_heads], sf.HEADS_ROWS, D ** -0.5, causal, lengths[few],
                          table[:, q_heads], of)
            for name, keys in (("dq", False), ("dk", True), ("dv", False)):
                within(rows_of(getattr(call, name)[few, :, q_heads if name == "dq" else k_heads], sf.HEADS_ROWS, keys), getattr(r, name), r.offs[name], name)
            one = r.offs["dtable"] - (UB if r.low else U) * r.dtable.abs() - 2.0 ** -120
            dtable[:, q_heads] += r.dtable
            off[:, q_heads] += one / (1 + UB) if r.low else one
            del r
    # (each turn's sums are rounded to fp32 once more, three times at most, of the 40 that `off` has for what is 20 otherwise)
    within(call.dtable.double(), dtable, off * (1 + UB) + UB * dtable.abs() + 2.0 ** -120 if dtype == torch.bfloat16 else off + U * dtable.abs() + 2.0 ** -120, "dtable")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 1, 2100, 8, 2, 128), (3, 5, 1030, 14, 2, 96), (2, 16, 700, 4, 4, 32), (1, 1, 5000, 7, 1, 80), (300, 2, 300, 2, 2, 40), (2, 15, 900, 6, 2, 64),
                                   (1, 70, 1500, 4, 2, 64)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("causal", [False, True], ids=["all", "causal"])
def test_few_queries_whose_keys_biases_differ(shape, dtype, causal):
    """A bucket drawn for each distance, some outside of the table: each key of a query has a bias of its own, each head another."""
    require_gpu()
    B, Tq, Tk, Hq, Hk, D = shape
    g = torch.Generator(device="cuda").manual_seed(Tk)
    lengths = torch.randint(0, Tk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    lengths[0] = Tk
    q, k, v, do = inputs(*shape, dtype, sf.HEADS_ROWS, seed=Tk, columns=True)
    table = (2.0 * torch.randn(50, Hq, generator=g, device="cuda")).to(dtype)
    of = torch.randint(-3, 53, (Tq + Tk - 1,), generator=g, device="cuda", dtype=torch.int32)
    call = Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, lengths, table, of).forward().backward()
    call.check()


@pytest.mark.parametrize("T,D", [(300, 128), (601, 104), (1100, 128)])
@pytest.mark.parametrize("causal", [False, True])
def test_wide_heads_whether_or_not_one_key_takes_most(T, D, causal):
    """All queries at once: dq within the bounds without the rounding of out where delta is formed anew, within those with it elsewhere."""
    require_gpu()
    q, k, v, do = inputs(2, T, T, 4 if T < 1000 else 16, 2, D, torch.bfloat16, sf.HEADS_ROWS, seed=T + D, spread=1.7)
    call = Call(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal).forward().backward()
    tight = RightDelta(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, None, None, None)
    wide = Reference(q, k, v, do, sf.HEADS_ROWS, D ** -0.5, causal, None, None, None)
    groups = torch.nn.functional.pad(call.stats[..., 1], (0, -T % 32), value=9.0).unflatten(2, (-1, 32))
    anew = ((groups > 0) & (groups < 2)).any(-1).repeat_interleave(32, -1)[:, :, :T, None]
    assert float(anew.float().mean()) > 0.25
    within(rows_of(call.dq, sf.HEADS_ROWS), wide.dq, torch.where(anew, tight.offs["dq"], wide.offs["dq"]), "dq")
