"""Host only: AdamW's calls refuse bad arguments before any launch, through the C ABI and through the binding."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2305_18513_amd import binding as sf

P, I, L, F, D = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_double


@pytest.fixture(scope="module")
def lib():
    if not sf.is_built():
        from paper_2305_18513_amd import build
        build.build_library(verbose=False)
    return sf.lib()


def _numel(*n):
    return (L * max(1, len(n)))(*n)


def test_workspace(lib):
    small, large = sf.adamw_workspace([5]), sf.adamw_workspace([5, 1 << 20])
    assert 0 < small < large and sf.adamw_workspace([]) >= 0
    out = C.c_size_t(0)
    assert lib.slimfit_adamw_workspace(I(1), _numel(1), None) == sf.ERR_INVALID_ARG
    assert lib.slimfit_adamw_workspace(I(-1), _numel(1), C.byref(out)) == sf.ERR_INVALID_ARG
    assert lib.slimfit_adamw_workspace(I(1), _numel(-1), C.byref(out)) == sf.ERR_INVALID_ARG
    assert lib.slimfit_adamw_workspace(I(1), _numel((1 << 33) + 1), C.byref(out)) == sf.ERR_UNSUPPORTED


def test_plan(lib):
    def call(w=1 << 20, g=1 << 21, m=1 << 22, v=1 << 23, ms=1 << 24, vs=1 << 25, copies=None, decay=0.1, bits=8, block=64, n=1000, w_dt=0, g_dt=0, ws=1 << 26,
             ws_bytes=1 << 20, layers=1):
        one = lambda p: (P * 1)(p)  # noqa: E731
        return lib.slimfit_adamw_plan(one(w), I(w_dt), one(g), I(g_dt), one(m), one(v), one(ms), one(vs), None if copies is None else one(copies),
                                      (F * 1)(decay), I(bits), I(block), _numel(n), I(layers), P(ws), C.c_size_t(ws_bytes), P(0))

    assert call(layers=0) == sf.OK
    for bad in (dict(w=0), dict(m=0), dict(v=0), dict(ms=0), dict(vs=0), dict(n=-1), dict(w_dt=2), dict(g_dt=-1), dict(decay=-0.1), dict(decay=float("nan")),
                dict(decay=float("inf")), dict(copies=1 << 27, w_dt=1), dict(layers=-1),
                dict(g=1 << 20), dict(m=(1 << 20) + 3984), dict(v=1 << 22), dict(copies=(1 << 20) + 16)):        # the last: shared memory
        assert call(**bad) == sf.ERR_INVALID_ARG, bad
    for bad in (dict(bits=4), dict(bits=16), dict(block=16), dict(block=96), dict(n=1 << 34)):
        assert call(**bad) == sf.ERR_UNSUPPORTED, bad
    for bad in (dict(w=(1 << 20) + 8), dict(g=(1 << 21) + 4), dict(m=(1 << 22) + 8), dict(v=(1 << 23) + 8), dict(ms=(1 << 24) + 2), dict(vs=(1 << 25) + 1),
                dict(copies=(1 << 27) + 8), dict(ws=(1 << 26) + 16)):
        assert call(**bad) == sf.ERR_ALIGNMENT, bad
    assert call(ws=0) == call(ws_bytes=64) == sf.ERR_WORKSPACE


def test_run(lib):
    def call(lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, step=1, floor=0.0, bits=32, block=0, n=1000, ws=1 << 26, ws_bytes=1 << 20, d=1 << 27, live=0, layers=1, w_dt=0):
        return lib.slimfit_adamw_run(_numel(n), I(layers), I(w_dt), I(0), I(bits), I(block), D(lr), D(b1), D(b2), D(eps), L(step), F(1.0), C.c_uint32(0), P(live),
                                     P(0), F(floor), P(d), P(ws), C.c_size_t(ws_bytes), P(0))

    assert call(layers=0) == sf.OK
    nan, inf = float("nan"), float("inf")
    for bad in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=nan),
                dict(eps=inf), dict(step=0), dict(step=1 << 32), dict(floor=-1.0), dict(floor=nan), dict(n=-1), dict(w_dt=7)):
        assert call(**bad) == sf.ERR_INVALID_ARG, bad
    assert call(bits=4) == call(bits=8, block=48) == call(n=1 << 34) == sf.ERR_UNSUPPORTED
    assert call(d=(1 << 27) + 2) == call(live=(1 << 27) + 1) == call(ws=(1 << 26) + 8) == sf.ERR_ALIGNMENT
    assert call(ws=0) == call(ws_bytes=8) == sf.ERR_WORKSPACE


def test_run_refuses_what_shares_memory(lib):
    """Distances over what the step reads, and a workspace over anything."""
    need = sf.adamw_workspace([1000] * 5)

    def call(ws=1 << 26, d=1 << 27, live=1 << 28, frozen=1 << 29):
        return lib.slimfit_adamw_run(_numel(*[1000] * 5), I(5), I(0), I(0), I(32), I(0), D(1e-3), D(0.9), D(0.999), D(1e-8), L(1), F(1.0), C.c_uint32(0), P(live),
                                     P(frozen), F(0.0), P(d), P(ws), C.c_size_t(need), P(0))

    for name in ("d", "live", "frozen"):
        for at in (1 << 26, (1 << 26) + need - 4):
            assert call(**{name: at}) == sf.ERR_INVALID_ARG, name
    assert call(d=(1 << 28) + 8) == call(live=(1 << 27) + 16) == call(d=(1 << 29) + 4) == call(frozen=(1 << 27) + 19) == sf.ERR_INVALID_ARG
    if not torch.cuda.is_available():                      # elsewhere the look-up of pointers says so
        for fine in (dict(), dict(d=(1 << 28) + 12), dict(frozen=(1 << 27) + 20), dict(live=1 << 29), dict(d=0, live=0, frozen=0)):
            assert call(**fine) not in (sf.ERR_INVALID_ARG, sf.OK), fine


def test_states(lib):
    def call(m=1 << 20, ms=1 << 21, v=1 << 22, vs=1 << 23, n=1000, block=64, mo=1 << 24, vo=1 << 25):
        return lib.slimfit_adamw_states(P(m), P(ms), P(v), P(vs), L(n), I(block), P(mo), P(vo), P(0))

    assert call(n=0) == sf.OK
    for bad in (dict(n=-1), dict(m=0), dict(ms=0), dict(v=0), dict(vs=0), dict(mo=0), dict(vo=0), dict(vo=1 << 24), dict(mo=1 << 20), dict(vo=(1 << 23) - 3984)):
        assert call(**bad) == sf.ERR_INVALID_ARG, bad
    assert call(block=48) == call(n=1 << 41) == sf.ERR_UNSUPPORTED
    for bad in (dict(m=(1 << 20) + 8), dict(v=(1 << 22) + 8), dict(mo=(1 << 24) + 8), dict(vo=(1 << 25) + 4), dict(ms=(1 << 21) + 2), dict(vs=(1 << 23) + 1)):
        assert call(**bad) == sf.ERR_ALIGNMENT, bad


def test_binding_refuses():
    t = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype)  # noqa: E731
    ws = torch.zeros(4096, dtype=torch.uint8)
    good = ([t(8)], [t(8)], [t(8)], [t(8)], None, None, [0.0], 32, 0, ws)
    for at, other in ((1, [t(9)]), (2, [t(7)]), (3, [t(8, torch.float64)]), (0, []), (6, []), (7, 8), (9, t(4))):
        with pytest.raises(ValueError):
            sf.adamw_plan(*good[:at], other, *good[at + 1:])
    with pytest.raises(ValueError):                        # not on the GPU
        sf.adamw_plan(*good) if torch.cuda.is_available() else sf._require(False)
    codes = [t(100, torch.uint8)]
    for scales in (None, [t(1)], [t(2, torch.float16)]):
        with pytest.raises(ValueError):
            sf.adamw_plan([t(100)], [None], codes, codes, scales, [t(2)], [0.0], 8, 64, ws)
    with pytest.raises(ValueError):
        sf.adamw_run(np.array([8]), 0, 0, 32, 0, 1e-3, 0.9, 0.999, 1e-8, 1, ws, d_out=t(0))
    with pytest.raises(ValueError):
        sf.adamw_run(np.array([8]), 0, 0, 32, 0, 1e-3, 0.9, 0.999, 1e-8, 1, ws, live=t(2))
    with pytest.raises(ValueError):
        sf.adamw_states(codes[0], t(1), codes[0], t(2), 64, t(100), t(100))


def test_plan_refuses_what_two_layers_share(lib):
    """A tensor, a state or the table's memory that two layers would write at once; gradients may be one tensor's."""
    base = dict(w=1 << 20, g=1 << 21, m=1 << 22, v=1 << 23, ms=1 << 24, vs=1 << 25)

    def call(second, bits=8, ws=1 << 26):
        first, n = dict(base), (L * 2)(4096, 4096)
        other = {k: x + (1 << 30) for k, x in first.items()}
        other.update(second)
        pair = lambda k: (P * 2)(first[k], other[k])  # noqa: E731
        return lib.slimfit_adamw_plan(pair("w"), I(0), pair("g"), I(0), pair("m"), pair("v"), pair("ms"), pair("vs"), P(0), (F * 2)(0.0, 0.0), I(bits), I(64), n,
                                      I(2), P(ws), C.c_size_t(64), P(0))

    assert call({}) == call(dict(g=base["g"])) == call(dict(w=(1 << 20) + 4 * 4096)) == sf.ERR_WORKSPACE          # (64 bytes are too few: the last check here)
    for bad in (dict(w=base["w"]), dict(w=(1 << 20) + 4 * 4096 - 16), dict(m=base["m"]), dict(v=base["m"] + 4080), dict(ms=base["vs"] + 252), dict(g=base["w"]),
                dict(vs=base["g"])):
        assert call(bad) == sf.ERR_INVALID_ARG, bad
    assert call({}, ws=base["m"]) == call({}, ws=(1 << 30) + base["g"]) == sf.ERR_INVALID_ARG
