"""AdamW on the GPU against the formulas on the CPU: states and codes bit for bit (rounded products and their rounded sum are
defined), weights and distances against 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2305_18513_amd import binding as sf
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

SIZES = [1, 7, 0, 255, 8192, 8193, 20011, 64, 3]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8)
SEED = 0x9234ABCD


def mix(x):
    x = x ^ (x >> np.uint32(16))
    x = x * np.uint32(0x6A09E667)
    x = x ^ (x >> np.uint32(15))
    x = x * np.uint32(0xBB67AE85)
    return x ^ (x >> np.uint32(16))


def dither(layer, n, step, seed=SEED):
    one = lambda v: np.array([v], dtype=np.uint32)  # noqa: E731
    key = mix(one(seed) ^ mix(one(step) ^ mix(one(layer + 1))))
    at = np.arange(n, dtype=np.uint32)
    word = mix(key + (at >> np.uint32(2))).astype(np.uint64)
    turn = (8 * (at & np.uint32(3))).astype(np.uint64)
    return ((((word << turn) | (word >> (32 - turn))) & 0xFFFFFFFF) >> 12).astype(np.uint32)


def runs_of(x, block):
    n = x.size
    return np.concatenate((x, np.zeros(-n % block, x.dtype))).reshape(-1, block)


def encode_m(m, block):
    r = runs_of(m, block)
    top = np.abs(r).max(1).astype(np.float32)
    with np.errstate(divide="ignore", over="ignore"):
        up = np.float32(448) / top
    fine = np.isfinite(up)
    by, scale = np.where(fine, up, 0).astype(np.float32), np.where(fine, top / np.float32(448), 0).astype(np.float32)
    code = torch.from_numpy(r * by[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    return code.reshape(-1)[: m.size], scale


def decode_m(code, scale, block):
    f = torch.from_numpy(runs_of(code, block)).view(torch.float8_e4m3fn).float().numpy() * scale[:, None]
    return f.reshape(-1)[: code.size]


def encode_v(v, block, noise):
    r = runs_of(v, block)
    top = np.maximum((r.max(1).view(np.uint32) >> 23).astype(np.int64) - 30, 1)
    code = ((r.view(np.uint32).astype(np.int64) + runs_of(noise.astype(np.int64), block)) >> 20) - 8 * top[:, None]
    code = np.where(r > 0, np.clip(code, 1, 255), 0).astype(np.uint8)
    return code.reshape(-1)[: v.size], (top << 23).astype(np.uint32).view(np.float32)


def decode_v(code, scale, block):
    c = runs_of(code, block).astype(np.uint32)
    bits = scale.view(np.uint32)[:, None] + (c << np.uint32(20))
    return np.where(c > 0, bits.view(np.float32), np.float32(0)).reshape(-1)[: code.size]


def widen(t):
    return t.float().cpu().numpy()


class Model:
    """Tensors as views between sentinels, on the GPU."""

    def __init__(self, sizes, w_dt, g_dt, bits, block, seed=0, copies=False):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.sizes, self.bits, self.block, self.w_dt, self.g_dt = sizes, bits, block, w_dt, g_dt
        self.kept = []

        def guarded(n, values):
            raw = torch.full((n + 64,), 77, dtype=values.dtype, device="cuda")
            raw[16 : 16 + n] = values
            self.kept.append((raw, n))
            return raw[16 : 16 + n]

        rand = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
        self.w = [guarded(n, (rand(n) * 0.1).to(w_dt)) for n in sizes]
        self.g = [guarded(n, (rand(n) * torch.exp(rand(n))).to(g_dt)) for n in sizes]
        if bits == 32:
            self.m, self.v = [guarded(n, rand(n)) for n in sizes], [guarded(n, rand(n).square()) for n in sizes]
            self.ms = self.vs = None
        else:
            self.m, self.v = ([guarded(n, torch.zeros(n, dtype=torch.uint8, device="cuda")) for n in sizes] for _ in range(2))
            self.ms, self.vs = ([guarded(-(-n // block), torch.zeros(-(-n // block), device="cuda")) for n in sizes] for _ in range(2))
        self.copies = [guarded(n, torch.zeros(n, dtype=torch.bfloat16, device="cuda")) for n in sizes] if copies else None
        self.decay = [0.1 if n > 64 else 0.0 for n in sizes]
        self.numel = np.array(sizes, dtype=np.int64)
        self.ws = torch.zeros(sf.adamw_workspace(sizes), dtype=torch.uint8, device="cuda")
        self.d = torch.full((len(sizes),), 5.0, device="cuda")

    def plan(self, grads=None, stream=None):
        sf.adamw_plan(self.w, self.g if grads is None else grads, self.m, self.v, self.ms, self.vs, self.decay, self.bits, self.block, self.ws, self.copies,
                      stream)

    def run(self, step, **more):
        args = dict(HYPER, step=step, workspace=self.ws, grad_factor=0.5, seed=SEED, floor=1e-3, d_out=self.d)
        args.update(more)
        sf.adamw_run(self.numel, sf._dt(torch.empty(0, dtype=self.w_dt)), sf._dt(torch.empty(0, dtype=self.g_dt)), self.bits, self.block, **args)

    def untouched_around(self):
        return all(bool((raw[:16] == 77).all()) and bool((raw[16 + n :] == 77).all()) for raw, n in self.kept)

    def tensors(self):
        return [t for each in (self.w, self.m, self.v, self.ms or [], self.vs or [], self.copies or []) for t in each]

    def expect(self, i, step):
        """(w in 64 bits before its rounding, size of its terms, m and v as they are stored, distance) after a step."""
        f32 = np.float32
        w, g = widen(self.w[i]), widen(self.g[i]) * f32(0.5)
        if self.bits == 32:
            m, v = widen(self.m[i]), widen(self.v[i])
        else:
            m = decode_m(self.m[i].cpu().numpy(), self.ms[i].cpu().numpy(), self.block)
            v = decode_v(self.v[i].cpu().numpy(), self.vs[i].cpu().numpy(), self.block)
        b1, b2 = HYPER["beta1"], HYPER["beta2"]
        m = m * f32(b1) + g * f32(1.0 - b1)
        v = v * f32(b2) + (g * f32(1.0 - b2)) * g
        assert m.dtype == v.dtype == np.float32
        w64 = w.astype(np.float64)
        d = -(HYPER["lr"] * float(f32(self.decay[i])) * w64 + HYPER["lr"] / (1 - b1 ** step) * m.astype(np.float64)
              / (np.sqrt(v.astype(np.float64) / (1 - b2 ** step)) + HYPER["eps"]))
        distance = float(np.mean(np.abs(d) / np.maximum(np.abs(w64), 1e-3))) if w.size else 0.0
        if self.bits == 32:
            held = ((m, None), (v, None))
        else:
            held = (encode_m(m, self.block), encode_v(v, self.block, dither(i, w.size, step)))
        size = np.abs(HYPER["lr"] * self.decay[i] * w64) + np.abs(d + HYPER["lr"] * float(f32(self.decay[i])) * w64)
        return w64 + d, size, held, distance


def check(model, before, i, w_dt):
    want, size, (m, v), distance = before
    # d: fifteen roundings at most on the way of either term (product, root, reciprocal step, sum, division); then the sum's
    bound = size * 15 * 2.0 ** -24 + np.abs(want) * 2.0 ** -24
    got = model.w[i].double().cpu().numpy()
    if w_dt == torch.bfloat16:
        bound = bound * (1 + 2.0 ** -8) + np.abs(want) * 2.0 ** -8
    assert np.all(np.abs(got - want) <= bound)
    assert np.array_equal(model.m[i].cpu().numpy(), m[0]) and np.array_equal(model.v[i].cpu().numpy(), v[0])
    if model.bits == 8:
        assert np.array_equal(model.ms[i].cpu().numpy(), m[1]) and np.array_equal(model.vs[i].cpu().numpy(), v[1])
    # a term: d's roundings and the division's, all terms >= 0, the sum in fp64, one rounding to fp32
    assert abs(float(model.d[i]) - distance) <= 18 * 2.0 ** -24 * distance + 1e-30
    if model.copies:
        assert torch.equal(model.copies[i], model.w[i].bfloat16())


@pytest.mark.parametrize("w_dt,g_dt", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16),
                                       (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("bits,block", [(32, 0), (8, 32), (8, 64), (8, 128), (8, 256)])
def test_steps(w_dt, g_dt, bits, block):
    require_gpu()
    model = Model(SIZES, w_dt, g_dt, bits, block, copies=w_dt == torch.float32)
    model.plan()
    for step in (1, 2, 3):
        before = [model.expect(i, step) for i in range(len(SIZES))]
        model.run(step)
        torch.cuda.synchronize()
        for i in range(len(SIZES)):
            check(model, before[i], i, w_dt)
    assert model.untouched_around()


@pytest.mark.parametrize("bits,block", [(32, 0), (8, 64)])
def test_frozen_layers_stay(bits, block):
    require_gpu()
    model = Model(SIZES, torch.float32, torch.float32, bits, block)
    mask = torch.tensor([i % 2 for i in range(len(SIZES))], dtype=torch.uint8, device="cuda")
    kept = [t.clone() for t in (*model.w, *model.m, *model.v)]
    grads = [None if i == 0 else g for i, g in enumerate(model.g)]
    model.plan(grads)
    before = {i: model.expect(i, 4) for i in (4, 6, 8)}
    model.run(4, frozen=mask)
    torch.cuda.synchronize()
    L = len(SIZES)
    for i in range(L):
        if i % 2 or i == 0:
            assert all(torch.equal(now, kept[k * L + i]) for k, now in enumerate((model.w[i], model.m[i], model.v[i])))
            assert float(model.d[i]) == 0.0
    for i, b in before.items():
        check(model, b, i, torch.float32)
    assert model.untouched_around()


def test_without_distances_and_no_layers():
    require_gpu()
    a, b = (Model(SIZES, torch.float32, torch.bfloat16, 8, 64, seed=3) for _ in range(2))
    for model, d in ((a, a.d), (b, None)):
        model.plan()
        model.run(1, d_out=d)
    assert all(torch.equal(x, y) for x, y in zip(a.tensors(), b.tensors())) and bool((b.d == 5.0).all())
    none = Model([], torch.float32, torch.float32, 32, 0)
    none.plan()
    none.run(1)


def test_stale_plan_touches_nothing():
    require_gpu()
    model = Model(SIZES, torch.float32, torch.float32, 32, 0)
    kept = [t.clone() for t in model.tensors()]
    model.run(1)                                           # never planned
    assert torch.isnan(model.d).all()
    model.plan()
    sf.adamw_run(model.numel, sf.F32, sf.BF16, 32, 0, 1e-3, 0.9, 0.999, 1e-8, 1, model.ws, d_out=model.d)      # another type
    assert torch.isnan(model.d).all()
    assert all(torch.equal(x, y) for x, y in zip(model.tensors(), kept))


@pytest.mark.parametrize("bits,block", [(32, 0), (8, 128)])
def test_captured_steps_follow_live(bits, block):
    """One captured step, replayed with the learning rate, step and factor of each step, between eager work, gives the eager bits."""
    require_gpu()
    a, b = (Model(SIZES, torch.float32, torch.float32, bits, block, seed=9) for _ in range(2))
    live = torch.zeros(3, device="cuda")
    a.plan()
    b.plan()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(1, live=live)
    lr = HYPER["lr"]
    for step, rate in ((1, lr), (2, lr), (3, lr / 2), (17, lr / 4), (1000003, lr)):
        rate32 = float(np.float32(rate))                   # a float is what live holds
        live.copy_(torch.tensor([rate32, step, 0.5]))
        graph.replay()
        b.run(step, lr=rate32)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a.tensors(), b.tensors())) and torch.equal(a.d, b.d)


def test_runs_on_streams_beside_each_other():
    require_gpu()
    alone = [Model(SIZES, torch.bfloat16, torch.bfloat16, 8, 64, seed=s) for s in (1, 2)]
    both = [Model(SIZES, torch.bfloat16, torch.bfloat16, 8, 64, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for model in alone:
        model.plan()
        for step in (1, 2, 3):
            model.run(step)
    torch.cuda.synchronize()
    for model, s in zip(both, streams):
        model.plan(stream=s.cuda_stream)
    for step in (1, 2, 3):
        for model, s in zip(both, streams):
            model.run(step, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        assert all(torch.equal(p, q) for p, q in zip(x.tensors(), y.tensors())) and torch.equal(x.d, y.d)


def test_gradients_that_are_not_finite_stay_in_their_block():
    require_gpu()
    model, other = (Model([1000], torch.float32, torch.float32, 8, 64, seed=5) for _ in range(2))
    model.g[0][130] = float("nan")
    model.g[0][700] = float("inf")
    for m in (model, other):
        m.plan()
        m.run(1)
    bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
    bad[[130, 700]] = True
    assert bool(torch.isnan(model.w[0][bad]).all()) and torch.equal(model.w[0][~bad], other.w[0][~bad])
    m_out, v_out = torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
    sf.adamw_states(model.m[0], model.ms[0], model.v[0], model.vs[0], 64, m_out, v_out)
    spoilt = (torch.arange(1000, device="cuda") // 64 == 130 // 64) | (torch.arange(1000, device="cuda") // 64 == 700 // 64)
    assert bool(torch.isfinite(m_out[~spoilt]).all()) and bool(torch.isfinite(v_out[~spoilt]).all()) and bool(torch.isnan(m_out[spoilt]).all())


@pytest.mark.parametrize("n", [1, 63, 64, 4099])
@pytest.mark.parametrize("block", [32, 256])
def test_states(n, block):
    require_gpu()
    g = torch.Generator().manual_seed(n)
    runs = -(-n // block)
    m, v = (torch.randint(0, 256, (n,), generator=g, dtype=torch.int16).to(torch.uint8) for _ in range(2))
    m[(m & 127) == 127] = 5                                # e4m3's NaN
    ms = torch.rand(runs, generator=g)
    vs = (torch.randint(1, 224, (runs,), generator=g, dtype=torch.int32) << 23).view(torch.float32)
    outs = [torch.full((n + 32,), 9.0, device="cuda") for _ in range(2)]
    sf.adamw_states(m.cuda(), ms.cuda(), v.cuda(), vs.cuda(), block, outs[0][:n], outs[1][:n])
    assert np.array_equal(outs[0][:n].cpu().numpy(), decode_m(m.numpy(), ms.numpy(), block))
    assert np.array_equal(outs[1][:n].cpu().numpy(), decode_v(v.numpy(), vs.numpy(), block))
    assert all(bool((o[n:] == 9.0).all()) for o in outs)


def test_a_v_decays_in_8_bits():
    """No gradient for 100 steps: each v in 8 bits moves by eighths, their mean by beta2 a step.  A step rounds up or down with a
    variance of at most (1/8)^2 * p, p = 0.008 being the steps' size over the code's: 0.011 a step, 0.11 after 100, over the mean of
    65536 4.4e-4 of it; seven of these are 0.0031."""
    require_gpu()
    model = Model([65536], torch.float32, torch.float32, 8, 64, seed=11)
    model.plan()
    model.run(1)
    out = [torch.empty(65536, device="cuda") for _ in range(2)]
    read = lambda: sf.adamw_states(model.m[0], model.ms[0], model.v[0], model.vs[0], 64, *out)  # noqa: E731
    read()
    start = out[1].double().clone()
    model.g[0].zero_()
    for step in range(2, 102):
        model.run(step)
    read()
    ratio = float((out[1].double() / start).mean())
    assert abs(ratio / 0.999 ** 100 - 1) < 0.0031


def test_offsets_past_32_bits():
    require_gpu()
    n = (1 << 30) + 4097
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of GPU memory")
    dev = "cuda"
    w, g = torch.full((n,), 0.5, device=dev), torch.full((n,), 1.0, dtype=torch.bfloat16, device=dev)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=dev) for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 256), device=dev) for _ in range(2))
    ws = torch.empty(sf.adamw_workspace([n]), dtype=torch.uint8, device=dev)
    d = torch.empty(1, device=dev)
    sf.adamw_plan([w], [g], [m], [v], [ms], [vs], [0.0], 8, 256, ws)
    sf.adamw_run(np.array([n]), sf.F32, sf.BF16, 8, 256, 0.25, 0.9, 0.999, 1e-8, 1, ws, seed=SEED, d_out=d)
    # the first step moves each weight by lr, to within its roundings
    for part in (w[:4096], w[n // 2 : n // 2 + 4096], w[-4097:]):
        assert float((part - 0.25).abs().max()) <= 0.25 * 15 * 2.0 ** -24
    assert abs(float(d) - 0.5) <= 18 * 2.0 ** -24
    noise = dither(0, 1 << 13, 1)                          # and the tail's codes are those of its own places
    at = np.arange(n - 4097, n, dtype=np.uint64)
    one = lambda x: np.array([x], dtype=np.uint32)  # noqa: E731
    word = mix(mix(one(SEED) ^ mix(one(1) ^ mix(one(1)))) + (at >> np.uint64(2)).astype(np.uint32)).astype(np.uint64)
    turn = 8 * (at & np.uint64(3))
    noise = ((((word << turn) | (word >> (32 - turn))) & 0xFFFFFFFF) >> 12).astype(np.uint32)
    v1 = np.full(4097, (np.float32(1.0) * np.float32(1.0 - 0.999)) * np.float32(1.0), np.float32)
    lead = (n - 4097) % 256
    code, _ = encode_v(np.concatenate((v1[:lead], v1)), 256, np.concatenate((noise[:lead] * 0, noise)))
    assert np.array_equal(v[-4097:].cpu().numpy(), code[lead:])
    assert math.isfinite(float(ms[-1]))


@pytest.mark.parametrize("bits,block", [(32, 0), (8, 256)])
def test_many_tensors_of_many_chunks(bits, block):
    """More tensors than are looked at together, empty ones among them, and chunks of the long kind (over 512 of 8192 elements)."""
    require_gpu()
    sizes = [3, 0, 0, 700, 8192, 1] * 24 + [4_400_003] + [0, 513, 0, 16385, 0] * 15
    model = Model(sizes, torch.float32, torch.bfloat16, bits, block)
    model.plan()
    looked_at = (0, 3, 4, 5, 60, 66, 143, 144, 146, 148, len(sizes) - 4, len(sizes) - 2)
    before = {i: model.expect(i, 2) for i in looked_at}
    kept = [t.clone() for t in model.w]
    model.run(2)
    torch.cuda.synchronize()
    for i, b in before.items():
        check(model, b, i, torch.float32)
    for i, n in enumerate(sizes):
        assert (n == 0 and float(model.d[i]) == 0.0) or (float(model.d[i]) > 0.0 and not torch.equal(kept[i], model.w[i]))
    assert model.untouched_around()


@pytest.mark.parametrize("eps", [1e-8, 1e-20, 1e-30])
def test_numbers_below_the_normal_ones(eps):
    """A v, an eps and weights at and below the type's least normal number, and a floor of 0: the distance's terms are those of the formula, a weight
    of 0 that moves makes it infinite, one that does not adds nothing."""
    require_gpu()
    tiny = np.float32(2.0 ** -126)
    w = [np.array([0.0, 1.0], np.float32), np.array([tiny / 4, 2.0, -tiny], np.float32), np.full(9, 0.25, np.float32), np.array([0.0, 0.5], np.float32)]
    g = [np.zeros(2, np.float32), np.array([2.0 ** -100, 1.0, -1.0], np.float32), np.linspace(1, 9, 9, dtype=np.float32) * np.float32(2.0 ** -66),
         np.array([1.0, 1.0], np.float32)]
    put = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    tw, tg = [put(x) for x in w], [put(x) for x in g]
    m, v = ([torch.zeros_like(t) for t in tw] for _ in range(2))
    numel = np.array([x.size for x in w], dtype=np.int64)
    ws, d = torch.zeros(sf.adamw_workspace(numel), dtype=torch.uint8, device="cuda"), torch.empty(4, device="cuda")
    sf.adamw_plan(tw, tg, m, v, None, None, [0.0] * 4, 32, 0, ws)
    sf.adamw_run(numel, sf.F32, sf.F32, 32, 0, 1e-2, 0.9, 0.999, eps, 1, ws, d_out=d)
    for i in range(4):
        m64 = m[i].double().cpu().numpy()                  # as they were stored: held products may be below the normal numbers
        v64 = v[i].double().cpu().numpy()
        assert np.array_equal(m[i].cpu().numpy(), g[i] * np.float32(1 - 0.9)) and np.array_equal(v[i].cpu().numpy(), (g[i] * np.float32(1 - 0.999)) * g[i])
        move = 1e-2 / 0.1 * m64 / (np.sqrt(v64 / (1 - 0.999)) + float(np.float32(eps)))
        want = w[i].astype(np.float64) - move
        # fifteen roundings of the move; a v below the normal numbers counts as 0 from an eps of 2^-40 on, a root of 2^-63 and so 2^-23 of the sum
        off = np.abs(move) * 17 * 2.0 ** -24 + np.abs(want) * 2.0 ** -24 + 2.0 ** -149
        assert np.all(np.abs(tw[i].double().cpu().numpy() - want) <= off)
    assert float(d[0]) == 0.0 and math.isinf(float(d[3]))
    terms = np.abs(1e-2 / 0.1 * m[2].double().cpu().numpy() / (np.sqrt(v[2].double().cpu().numpy() / (1 - 0.999)) + float(np.float32(eps)))) / 0.25
    assert abs(float(d[2]) - terms.mean()) <= 20 * 2.0 ** -24 * terms.mean() + 2.0 ** -149


@pytest.mark.parametrize("eps", [1e-10, 1e-11, 1e-12, 9.2e-13, 9e-13])
@pytest.mark.parametrize("beta2", [0.999, 1.0 - 1e-6, 0.5])
@pytest.mark.parametrize("live", [False, True])
def test_an_eps_near_what_a_root_below_the_normal_numbers_adds(eps, beta2, live):
    """At the first step a root of v counts 1 / sqrt(1 - beta2) times, up to a thousand here, beside eps.  Weights of 0, so that the move itself is
    seen: fifteen roundings, and one of the weight."""
    require_gpu()
    tiny = 2.0 ** -126
    g = np.sqrt(np.array([0.9, 0.99, 0.5, 0.1, 0.01, 1.01, 4.0, 1e6]) * tiny / (1 - beta2)).astype(np.float32)
    w, grad = torch.zeros(g.size, device="cuda"), torch.from_numpy(g).cuda()
    m, v = torch.zeros_like(w), torch.zeros_like(w)
    ws, d = torch.zeros(sf.adamw_workspace([g.size]), dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
    sf.adamw_plan([w], [grad], [m], [v], None, None, [0.0], 32, 0, ws)
    now = torch.tensor([0.25, 1.0, 1.0], device="cuda") if live else None
    sf.adamw_run([g.size], sf.F32, sf.F32, 32, 0, 0.25, 0.9, beta2, eps, 1, ws, live=now, floor=1.0, d_out=d)
    m64, v64 = m.double().cpu().numpy(), v.double().cpu().numpy()
    assert np.array_equal(v.cpu().numpy(), (g * np.float32(1 - beta2)) * g) and int((v64 < tiny).sum()) >= 4
    move = 0.25 / 0.1 * m64 / (np.sqrt(v64 / (1 - beta2)) + float(np.float32(eps)))
    assert np.all(np.abs(w.double().cpu().numpy() + move) <= np.abs(move) * 16 * 2.0 ** -24 + 2.0 ** -149)
    assert abs(float(d) - move.mean()) <= 18 * 2.0 ** -24 * move.mean() + 2.0 ** -149


@pytest.mark.parametrize("block", [32, 64, 256])
@pytest.mark.parametrize("bad", [math.nan, -math.nan, math.inf, -math.inf, 3e21])
def test_a_v_that_is_not_finite_is_its_whole_blocks(bad, block):
    """In 8 bits a block's v are all NaN then (a scale for so large a number has no codes for the others), those without a gradient too, and the
    next step's weights with them; the blocks beside it go on.  A gradient of 3e21 is finite, its v' (9e39) is not."""
    require_gpu()
    n = 5 * block + 3
    model, other = (Model([n], torch.float32, torch.float32, 8, block, seed=5) for _ in range(2))
    here = torch.arange(n, device="cuda") // block == 2
    for m in (model, other):
        m.g[0][2 * block + 1 :: 7] = 0.0
    model.g[0][2 * block + 5] = bad
    outs = [torch.empty(n, device="cuda") for _ in range(4)]
    for step in (1, 2):
        for m in (model, other):
            m.plan()
            m.run(step, grad_factor=1.0)
        for m, (m_out, v_out) in ((model, outs[:2]), (other, outs[2:])):
            sf.adamw_states(m.m[0], m.ms[0], m.v[0], m.vs[0], block, m_out, v_out)
        assert bool(torch.isnan(outs[1][here]).all())
        assert bool(torch.isnan(outs[0][here]).all()) or bad == 3e21
        assert torch.equal(outs[0][~here], outs[2][~here]) and torch.equal(outs[1][~here], outs[3][~here])
        assert torch.equal(model.w[0][~here], other.w[0][~here])
    assert bool(torch.isnan(model.w[0][here]).all())
    assert model.untouched_around()
