"""Host only: the calls around a decoder layer's cached activations refuse bad arguments before any launch, through the C ABI
and through the binding."""
import ctypes as C

import pytest
import torch

from paper_2305_18513_amd import binding as sf

P, I, L, F = C.c_void_p, C.c_int32, C.c_int64, C.c_float


@pytest.fixture(scope="module")
def lib():
    if not sf.is_built():
        from paper_2305_18513_amd import build
        build.build_library(verbose=False)
    return sf.lib()


def test_gated(lib):
    def fwd(x=1 << 20, dt=0, rows=4, width=64, act=0, mode=1, bits=8, block=32, fb=0, y=1 << 24, codes=1 << 25, scales=1 << 26):
        return lib.slimfit_gated_quant_pack(P(x), I(dt), L(rows), L(width), I(act), I(mode), I(bits), I(block), I(fb), P(y), P(codes), P(scales), P(0))

    def bwd(codes=1 << 25, scales=1 << 26, rows=4, width=64, act=0, mode=1, bits=8, block=32, fb=0, dy=1 << 20, dx=1 << 24, dt=0):
        return lib.slimfit_gated_backward_dequant(P(codes), P(scales), L(rows), L(width), I(act), I(mode), I(bits), I(block), I(fb), P(dy), P(dx), I(dt),
                                                  P(0))

    for call in (fwd, bwd):
        assert call(rows=0) == sf.OK and call(width=0) == sf.OK
        for bad in (dict(rows=-1), dict(width=-32), dict(dt=2), dict(act=2), dict(act=-1), dict(mode=2), dict(codes=0), dict(scales=0)):
            assert call(**bad) == sf.ERR_INVALID_ARG, bad
        for bad in (dict(bits=5), dict(block=48), dict(width=96, block=64), dict(mode=0, fb=33), dict(mode=0, width=6), dict(dt=1, mode=0, width=12),
                    dict(width=1 << 25), dict(rows=1 << 40)):
            assert call(**bad) == sf.ERR_UNSUPPORTED, bad
        assert call(codes=(1 << 25) + 8) == sf.ERR_ALIGNMENT and call(scales=(1 << 26) + 4) == sf.ERR_ALIGNMENT
    assert bwd(bits=0) == sf.ERR_UNSUPPORTED
    assert fwd(x=0) == fwd(y=0) == bwd(dy=0) == bwd(dx=0) == sf.ERR_INVALID_ARG
    assert fwd(x=(1 << 20) + 4) == fwd(y=(1 << 24) + 8) == bwd(dy=(1 << 20) + 8) == bwd(dx=(1 << 24) + 8) == sf.ERR_ALIGNMENT
    assert fwd(y=(1 << 20) + 4 * 128 * 4 - 16) == fwd(y=(1 << 20) - 16) == sf.ERR_INVALID_ARG       # shared memory
    assert bwd(dx=1 << 20) == sf.ERR_INVALID_ARG


def _heads(lib, back):
    def call(dt=0, batch=2, tokens=8, q_heads=4, kv_heads=2, dim=64, gq=1 << 20, gk=1 << 21, eps=1e-6, table=1 << 22, places=16, rotary=32, pairing=0,
             ids=0, bits=8, block=32, q=1 << 24, kt=1 << 25, v=1 << 26, qkv=1 << 27, rstd=1 << 28, codes=1 << 29, scales=1 << 30, dgq=1 << 31,
             dgk=(1 << 31) + 256, ws=1 << 32, ws_bytes=1 << 20):
        sizes = (L(batch), I(tokens), I(q_heads), I(kv_heads), I(dim))
        turn = (P(table), I(places), I(rotary), I(pairing), P(ids), F(0.5))
        if back:
            return lib.slimfit_heads_norm_rotate_backward(P(q), P(kt), P(v), P(1 << 33), P(codes), P(scales), I(bits), I(block), P(rstd), I(dt), *sizes, P(gq),
                                                          P(gk), *turn, P(qkv), P(dgq), P(dgk), P(ws), C.c_size_t(ws_bytes), P(0))
        return lib.slimfit_heads_norm_rotate_forward(P(qkv), I(dt), *sizes, P(gq), P(gk), F(eps), *turn, I(bits), I(block), P(q), P(kt), P(v), P(rstd),
                                                     P(codes), P(scales), P(0))
    return call


@pytest.mark.parametrize("back", [False, True])
def test_heads(lib, back):
    call = _heads(lib, back)
    none = dict(dgq=0, dgk=0)
    assert call(batch=0, **none) == sf.OK and call(tokens=0, **none) == sf.OK
    for bad in (dict(dt=2), dict(batch=-1), dict(tokens=-1), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=3), dict(dim=0), dict(gk=0), dict(rotary=-8),
                dict(rotary=72), dict(places=-1), dict(pairing=2), dict(places=7), dict(table=0), dict(q=0), dict(kt=0), dict(v=0), dict(qkv=0),
                dict(rstd=0), dict(codes=0), dict(scales=0), dict(gq=0, gk=0, **none)):
        assert call(**bad) == sf.ERR_INVALID_ARG, bad
    for bad in (dict(dim=66, bits=0), dict(dim=260, bits=0), dict(dt=1, dim=12, bits=0, rotary=0), dict(dt=1, rotary=24), dict(rotary=12), dict(bits=5),
                dict(block=48), dict(dim=96, block=64), dict(batch=1 << 31, tokens=1), dict(batch=1 << 20, tokens=1 << 12, places=1 << 12)):
        assert call(**bad) == sf.ERR_UNSUPPORTED, bad
    for bad in (dict(q=(1 << 24) + 8), dict(kt=(1 << 25) + 8), dict(v=(1 << 26) + 4), dict(qkv=(1 << 27) + 4), dict(rstd=(1 << 28) + 2),
                dict(codes=(1 << 29) + 4), dict(scales=(1 << 30) + 4), dict(table=(1 << 22) + 4), dict(ids=(1 << 23) + 2), dict(gq=(1 << 20) + 4)):
        assert call(**bad) == sf.ERR_ALIGNMENT, bad
    assert call(q=(1 << 27) + 4096) == call(kt=1 << 27) == call(v=(1 << 27) + 16) == sf.ERR_INVALID_ARG      # shared memory
    if back:
        assert call(dgk=0) == sf.ERR_INVALID_ARG
        assert call(ws=0) == sf.ERR_WORKSPACE and call(ws_bytes=64) == sf.ERR_WORKSPACE
        assert call(ws=(1 << 32) + 8) == sf.ERR_ALIGNMENT and call(dgq=(1 << 31) + 4) == sf.ERR_ALIGNMENT
    else:
        assert call(eps=-1.0) == call(eps=float("nan")) == sf.ERR_INVALID_ARG
        assert call(v=1 << 24) == call(kt=1 << 26) == sf.ERR_INVALID_ARG


def test_heads_workspace(lib):
    assert sf.heads_norm_rotate_workspace(torch.float32, 0, 8, 4, 2, 64) == 0
    assert sf.heads_norm_rotate_workspace(torch.float32, 2, 8, 4, 2, 64) >= 6 * 64 * 4
    for bad in ((2, 8, 4, 3, 64), (-1, 8, 4, 2, 64), (2, 8, 4, 2, 66), (2, 8, 4, 2, 300)):
        with pytest.raises(sf.SlimfitError):
            sf.heads_norm_rotate_workspace(torch.float32, *bad)


def test_weight_gradient(lib):
    def call(dy=1 << 20, dt=0, codes=1 << 24, scales=1 << 25, bits=8, block=32, M=16, N=8, K=64, dw=1 << 26, ws=0, ws_bytes=0):
        return lib.slimfit_weight_grad_dequant(P(dy), I(dt), P(codes), P(scales), I(bits), I(block), L(M), L(N), L(K), P(dw), P(ws), C.c_size_t(ws_bytes),
                                               P(0))

    assert call(N=0) == sf.OK and call(K=0) == sf.OK
    for bad in (dict(dt=2), dict(M=-1), dict(N=-1), dict(K=-64), dict(dy=0), dict(codes=0), dict(scales=0), dict(dw=0), dict(dw=1 << 20), dict(dw=1 << 24),
                dict(dw=(1 << 25) - 16)):
        assert call(**bad) == sf.ERR_INVALID_ARG, bad
    for bad in (dict(bits=6), dict(bits=0), dict(block=48), dict(block=64, K=96), dict(N=(1 << 20) + 1), dict(K=1 << 21), dict(M=(1 << 40) + 1)):
        assert call(**bad) == sf.ERR_UNSUPPORTED, bad
    for bad in (dict(dy=(1 << 20) + 8), dict(codes=(1 << 24) + 4), dict(scales=(1 << 25) + 4), dict(dw=(1 << 26) + 4)):
        assert call(**bad) == sf.ERR_ALIGNMENT, bad
    need = sf.weight_grad_dequant_workspace(torch.float32, 32, 100000, 8, 64)
    assert need > 0 and sf.weight_grad_dequant_workspace(torch.float32, 32, 100000, 0, 64) == 0
    far = dict(M=100000, dy=1 << 40, codes=1 << 41, scales=1 << 42)
    assert call(**far) == call(ws=1 << 43, ws_bytes=need - 1, **far) == sf.ERR_WORKSPACE
    assert call(ws=(1 << 43) + 8, ws_bytes=need, **far) == sf.ERR_ALIGNMENT
    for bad in ((torch.float32, 48, 4, 4, 96), (torch.float32, 32, -1, 4, 64), (torch.float32, 32, 4, 1 << 21, 64)):
        with pytest.raises(sf.SlimfitError):
            sf.weight_grad_dequant_workspace(*bad)


def test_binding_wants_the_gpu_and_sizes_that_agree(lib):
    """Tensors of the host are refused, also where everything else agrees; what does not agree is refused before that."""
    z = torch.zeros
    codes, scales = z(512, dtype=torch.uint8), z(16)
    for call, text in ((lambda: sf.gated_quant_pack(z(4, 128), 0, 1, 8, 32, 0, z(4, 64), codes, scales), "current GPU"),
                       (lambda: sf.gated_quant_pack(z(4, 128), 0, 1, 8, 32, 0, z(4, 32), codes, scales), "agree"),
                       (lambda: sf.gated_backward_dequant(codes, scales, 0, 1, 8, 32, 0, z(4, 64), z(4, 128)), "current GPU"),
                       (lambda: sf.gated_backward_dequant(codes[1:], scales, 0, 1, 8, 32, 0, z(4, 64), z(4, 128)), "agree"),
                       (lambda: sf.weight_grad_dequant(z(4, 8), codes, scales, 8, 32, z(8, 128)), "current GPU"),
                       (lambda: sf.weight_grad_dequant(z(4, 8), codes, scales, 8, 32, z(7, 128)), "agree"),
                       (lambda: sf.weight_grad_dequant(z(4, 8), codes, scales[1:], 8, 32, z(8, 128)), "agree"),
                       (lambda: sf.heads_norm_rotate_forward(z(2, 3, 64), None, None, 0.0, None, 0, None, 1.0, 0, 0, z(2, 2, 3, 16), z(2, 1, 16, 3),
                                                             z(2, 1, 3, 16), None, None, None), "current GPU"),
                       (lambda: sf.heads_norm_rotate_forward(z(2, 3, 64), None, None, 0.0, None, 0, None, 1.0, 0, 0, z(2, 2, 3, 16), z(2, 1, 3, 16),
                                                             z(2, 1, 3, 16), None, None, None), "agree"),
                       (lambda: sf.heads_norm_rotate_backward(z(2, 2, 3, 16), z(2, 1, 16, 3), z(2, 1, 3, 16), None, None, None, 0, 0, None, None, None, None, 0,
                                                              None, 1.0, z(2, 3, 64)), "current GPU"),
                       (lambda: sf.heads_norm_rotate_backward(z(2, 2, 3, 16), z(2, 1, 16, 3), z(2, 1, 3, 16), None, None, None, 0, 0, z(18), z(16), z(16), None, 0,
                                                              None, 1.0, z(2, 3, 64)), "agree")):
        with pytest.raises(ValueError, match=text):
            call()


def test_rotary_table():
    t = sf.rotary_table(5, 8, 10000.0, "cpu")
    assert t.shape == (5, 8) and t.dtype == torch.float32
    angle = torch.arange(5).double()[:, None] * torch.tensor([1.0, 0.1, 0.01, 0.001]).double()
    assert torch.allclose(t.double(), torch.cat((angle.cos(), angle.sin()), 1), rtol=0, atol=2.0 ** -24)


@pytest.mark.parametrize("grad", [True, False])
def test_wrappers_keep_nothing_where_gradients_are_off(grad, monkeypatch):
    """Trainable gains, weights and inputs under no_grad: the calls are asked for no cache and nothing is quantised."""
    from paper_2305_18513_amd import autograd as ag

    asked = []
    monkeypatch.setattr(ag.sf, "gated_quant_pack", lambda x, act, mode, bits, *rest: asked.append(bits))
    monkeypatch.setattr(ag.sf, "heads_norm_rotate_forward", lambda *a: asked.append(a[8]))
    monkeypatch.setattr(ag.sf, "quant_pack", lambda x, mode, bits, *rest: asked.append(bits))

    def leaf(*shape):
        return torch.zeros(*shape, requires_grad=True)

    with torch.set_grad_enabled(grad):
        outs = [ag.GatedFunction.apply(leaf(2, 128), sf.ACT_SILU, 8, 32),
                ag.HeadsNormRotateFunction.apply(torch.zeros(1, 2, 256), leaf(64), leaf(64), 2, 1, None)[0],
                ag.LinearFunction.apply(torch.zeros(4, 64), leaf(8, 64), leaf(8))]
    assert asked == ([8, 8, 8] if grad else [0, 0])
    assert all(o.requires_grad == grad for o in outs)
