"""Host only: the attention calls refuse bad arguments before any launch, through the C ABI and through the binding."""
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


def _call(lib, back):
    def call(q=1 << 30, k=1 << 31, v=1 << 32, dt=0, layout=0, q_row=256, k_row=128, v_row=128, batch=2, tq=10, tk=20, hq=4, hk=2, dim=64, scale=0.125, causal=0,
             lengths=0, table=0, buckets=0, of=0, out=1 << 33, stats=1 << 34, ws=1 << 35, ws_bytes=1 << 24, dout=1 << 36, dq=1 << 37, dk=1 << 38, dv=1 << 39,
             dq_row=256, dk_row=128, dv_row=128, dtable=0):
        one = (P(q), P(k), P(v), I(dt), I(layout), L(q_row), L(k_row), L(v_row), L(batch), I(tq), I(tk), I(hq), I(hk), I(dim), F(scale), I(causal), P(lengths),
               P(table), I(buckets), P(of), P(out), P(stats))
        if back:
            return lib.slimfit_attention_backward(P(dout), *one, P(dq), P(dk), P(dv), L(dq_row), L(dk_row), L(dv_row), P(dtable), P(ws), C.c_size_t(ws_bytes), P(0))
        return lib.slimfit_attention_forward(*one, P(ws), C.c_size_t(ws_bytes), P(0))
    return call


@pytest.mark.parametrize("back", [False, True])
def test_calls(lib, back):
    call = _call(lib, back)
    if not back:
        assert call(batch=0) == call(tq=0) == sf.OK
    nan, inf = float("nan"), float("inf")
    for bad in (dict(dt=2), dict(layout=2), dict(layout=-1), dict(batch=-1), dict(tq=-1), dict(tk=-1), dict(hq=0), dict(hk=0), dict(hq=3), dict(dim=0), dict(dim=-8),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf), dict(q_row=248), dict(k_row=120), dict(v_row=64), dict(q=0), dict(k=0), dict(v=0),
                dict(out=0), dict(stats=0), dict(table=1 << 20, buckets=0, of=1 << 21), dict(table=1 << 20, buckets=4, of=0), dict(table=1 << 20, buckets=-1, of=1 << 21)):
        assert call(**bad) == sf.ERR_INVALID_ARG, bad
    for bad in (dict(dim=66), dict(dim=132, q_row=1024, k_row=512, v_row=512, dq_row=1024, dk_row=512, dv_row=512), dict(dt=1, dim=20), dict(tq=(1 << 28) + 1),
                dict(tk=(1 << 28) + 1), dict(batch=1 << 25), dict(batch=1 << 20), dict(table=1 << 20, buckets=1025, of=1 << 21), dict(q_row=(1 << 20) + 8),
                dict(hq=1 << 16, hk=1)):
        assert call(**bad) == sf.ERR_UNSUPPORTED, bad
    for bad in (dict(q=(1 << 30) + 8), dict(k=(1 << 31) + 4), dict(v=(1 << 32) + 2), dict(out=(1 << 33) + 8), dict(stats=(1 << 34) + 8), dict(q_row=258), dict(k_row=129),
                dict(lengths=(1 << 20) + 2), dict(table=(1 << 20) + 2, buckets=4, of=1 << 21), dict(table=1 << 20, buckets=4, of=(1 << 21) + 1)):
        assert call(**bad) == sf.ERR_ALIGNMENT, bad
    assert call(layout=1, ws=0) == call(layout=1, ws_bytes=64) == sf.ERR_WORKSPACE and call(layout=1, ws=(1 << 35) + 8) == sf.ERR_ALIGNMENT
    row = 1024                                             # columns of the same rows share nothing, a column more does
    if back:
        assert call(dq=1 << 30) == call(dk=1 << 31) == call(dv=(1 << 38) + 512) == call(dq=1 << 36) == call(dk=1 << 33) == sf.ERR_INVALID_ARG
        base = 1 << 40
        apart = dict(dq=base, dk=base + 4 * 256, dv=base + 4 * 384, dq_row=row, dk_row=row, dv_row=row, tk=10)
        assert call(**apart, ws=0) == sf.ERR_WORKSPACE     # all but the workspace is fine
        assert call(**dict(apart, dk=base + 4 * 252), ws=0) == call(**dict(apart, dv=base + 4 * 380), ws=0) == sf.ERR_INVALID_ARG
        assert call(**dict(apart, dq_row=512), ws=0) == sf.ERR_INVALID_ARG
        assert call(dtable=1 << 20) == sf.ERR_INVALID_ARG  # without a table
        bias = dict(table=1 << 20, buckets=4, of=1 << 21)
        assert call(**bias, dtable=1 << 20) == call(**bias, dtable=1 << 37) == sf.ERR_INVALID_ARG and call(**bias, dtable=(1 << 22) + 2) == sf.ERR_ALIGNMENT
        assert call(**bias, dtable=1 << 22, ws_bytes=256) == sf.ERR_WORKSPACE
        assert call(dq_row=128) == sf.ERR_INVALID_ARG and call(dv_row=130) == sf.ERR_ALIGNMENT
    else:
        assert call(out=1 << 30) == call(stats=(1 << 31) + 16) == call(stats=1 << 33) == sf.ERR_INVALID_ARG


@pytest.mark.parametrize("back", [False, True])
def test_calls_refuse_what_shares_memory(lib, back):
    """Outputs over the lengths, the table or the distances, and a workspace over anything: part of either is enough."""
    call = _call(lib, back)
    few = dict(lengths=1 << 20, table=1 << 21, buckets=4, of=1 << 22, layout=1)           # 8 bytes, 64, 116
    small = dict(few, ws_bytes=64)
    assert call(**small) == sf.ERR_WORKSPACE                # all but the workspace is fine
    outs = ("dq", "dk", "dv", "dtable") if back else ("out", "stats")
    for name in outs:
        for at in (1 << 20, 1 << 21, (1 << 21) + 48, 1 << 22, (1 << 22) + 112):
            assert call(**dict(small, **{name: at})) == sf.ERR_INVALID_ARG, (name, at)
        assert call(**dict(small, **{name: (1 << 22) + 128})) == sf.ERR_WORKSPACE, name
        # (what is not read may be anywhere)
        assert call(**dict(small, table=0, **{name: 1 << 22})) == (sf.ERR_INVALID_ARG if name == "dtable" else sf.ERR_WORKSPACE)
    need = sf.attention_workspace(torch.float32, sf.HEADS_APART, 2, 10, 20, 4, 2, 64, back, back)
    full = dict(few, ws=1 << 35, ws_bytes=need, **(dict(dtable=1 << 23) if back else {}))
    for name in outs + ("q", "k", "v", "lengths", "table", "of") + (("dout", "out", "stats") if back else ()):
        for at in (1 << 35, (1 << 35) + need - 16):
            assert call(**dict(full, **{name: at})) == sf.ERR_INVALID_ARG, name
    if not torch.cuda.is_available():                       # elsewhere the look-up of pointers says so
        assert call(**full) not in (sf.ERR_INVALID_ARG, sf.ERR_WORKSPACE, sf.ERR_ALIGNMENT, sf.OK)
        assert call(**dict(full, q=(1 << 35) + need)) not in (sf.ERR_INVALID_ARG, sf.OK)


@pytest.mark.parametrize("back", [False, True])
def test_calls_refuse_scales_without_a_logarithm_of_base_2(lib, back):
    call = _call(lib, back)
    for scale in (2.0 ** 127, 3e38):
        assert call(scale=scale) == sf.ERR_INVALID_ARG
    if not torch.cuda.is_available():
        for scale in (1.7e38, 1e-38, 2.0 ** -149):
            assert call(scale=scale) not in (sf.ERR_INVALID_ARG, sf.OK)


def test_workspace(lib):
    size = lambda **kw: sf.attention_workspace(**dict(dict(dtype=torch.bfloat16, layout=sf.HEADS_ROWS, batch=2, q_tokens=100, k_tokens=50, q_heads=4,  # noqa: E731
                                                           kv_heads=2, head_dim=64), **kw))
    assert size() == 0 and size(layout=sf.HEADS_APART) >= 2 * 2 * 50 * 64 * 2
    back = size(backward=True)
    assert back >= 2 * 4 * 100 * 12 and size(backward=True, with_dtable=True) > back
    out = C.c_size_t(0)
    assert lib.slimfit_attention_workspace(I(0), I(0), L(1), I(1), I(1), I(1), I(1), I(64), I(0), I(0), None) == sf.ERR_INVALID_ARG
    assert lib.slimfit_attention_workspace(I(0), I(0), L(1), I(1), I(1), I(1), I(1), I(130), I(0), I(0), C.byref(out)) == sf.ERR_UNSUPPORTED


def test_the_workspace_of_shared_out_tiles():
    """The sums by distance of shares: what they write, not a whole row of keys for each of up to 64."""
    size = lambda table: sf.attention_workspace(torch.bfloat16, sf.HEADS_ROWS, 1, 128, 1 << 20, 1, 1, 128, table, True)  # noqa: E731
    # 64 shares of 256 tiles, 4 waves' rows of 257 * 64 floats each; 8 shares of the sums over 128 + 2^20 distances
    assert 0 < size(True) - size(False) <= 64 * 4 * 257 * 64 * 4 + 8 * (128 + (1 << 20)) * 4 + 512


def test_the_tables_gradient_takes_memory_by_the_length():
    """Not by the pairs: 256 MB, or 32 KB a key, or 16 bytes a key, sequence and head, and up to 33 sums for each head and distance."""
    for B, T, H in ((1, 65536, 16), (16, 4096, 16), (16, 16384, 16), (300, 1024, 12), (1, 1 << 20, 1), (4000, 500, 16)):
        for dtype in (torch.float32, torch.bfloat16):
            size = lambda table: sf.attention_workspace(dtype, sf.HEADS_ROWS, B, T, T, H, H, 64, table, True)  # noqa: E731, B023
            assert size(True) - size(False) <= max(256 << 20, (T + 127) * max(32768, 16 * B * H)) + 33 * H * 2 * T * 4 + 512, (B, T, H)


def test_distance_buckets():
    one = sf.distance_buckets(5, 5, 8, 16, both_ways=False, device="cpu")
    assert one.dtype == torch.int32 and one.tolist() == [4, 3, 2, 1, 0, 0, 0, 0, 0]
    both = sf.distance_buckets(40, 40, 8, 16, device="cpu")
    assert both.tolist()[39] == 0 and both.tolist()[40] == 5 and both.tolist()[38] == 1 and both[0] == 3 and both[-1] == 7
    for n in (1, 2, 3, 7, 32):
        for ways in (False, True):
            b = sf.distance_buckets(300, 200, n, 64, ways, device="cpu")
            assert b.numel() == 499 and int(b.min()) >= 0 and int(b.max()) < n
            past = b[:300].flip(0)                         # distance 0, -1, ...: never falls
            assert bool((past[1:] >= past[:-1]).all())


@pytest.mark.parametrize("buckets", [1, 2, 7, 32])
def test_distances_stand_where_the_causal_order_does(buckets):
    """The last tokens over all keys, and keys over which some queries come too early, have the buckets of the same rows and columns of a whole pass."""
    T = 300
    whole = sf.distance_buckets(T, T, buckets, 128, both_ways=False, device="cpu")
    row = lambda of, i, Tq, Tk: of[torch.arange(Tk) - i + Tq - 1]  # noqa: E731
    for n in (1, 3, 16, 299):
        few = sf.distance_buckets(n, T, buckets, 128, both_ways=False, device="cpu")
        assert few.numel() == n + T - 1
        for i in range(n):
            assert torch.equal(row(few, i, n, T), row(whole, T - n + i, T, T))
        late = sf.distance_buckets(T, n, buckets, 128, both_ways=False, device="cpu")     # the last n keys
        for i in range(0, T, 7):
            assert torch.equal(row(late, i, T, n), row(whole, i, T, T)[T - n :])
    assert sf.distance_buckets(1, 4096, 32, 128, both_ways=False, device="cpu").unique().numel() == 32
    both = sf.distance_buckets(T, T, buckets, 128, device="cpu")                          # both ways: on request
    few = sf.distance_buckets(4, T, buckets, 128, device="cpu", first_query=T - 4)
    assert all(torch.equal(row(few, i, 4, T), row(both, T - 4 + i, T, T)) for i in range(4))
    few = sf.distance_buckets(4, T, buckets, 128, device="cpu")
    assert all(torch.equal(row(few, i, 4, T), row(both, i, T, T)) for i in range(4))


def test_binding_refuses():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    q, k, v, out, stats = z(2, 5, 4, 8), z(2, 7, 2, 8), z(2, 7, 2, 8), z(2, 5, 4, 8), z(2, 4, 5, 2)
    good = dict(q=q, k=k, v=v, layout=sf.HEADS_ROWS, scale=1.0, causal=False, lengths=None, table=None, bucket_of=None, out=out, stats=stats)
    table, of = z(3, 4), z(11, dtype=torch.int32)
    for bad in (dict(k=z(2, 7, 3, 8)), dict(v=z(2, 6, 2, 8)), dict(out=z(2, 4, 5, 8)), dict(stats=z(2, 4, 5)), dict(out=z(2, 5, 4, 8, dtype=torch.bfloat16)),
                dict(q=z(2, 5, 4, 8, dtype=torch.bfloat16)), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(lengths=z(2)), dict(layout=7),
                dict(lengths=z(1, dtype=torch.int32)), dict(table=table), dict(table=table, bucket_of=z(10, dtype=torch.int32)), dict(table=z(3, 3), bucket_of=of),
                dict(table=table, bucket_of=of.long()), dict(layout=sf.HEADS_APART), dict(q=q[0])):
        with pytest.raises(ValueError):
            sf.attention_forward(**dict(good, **bad))
    back = dict(good, dout=z(2, 5, 4, 8), dq=z(2, 5, 4, 8), dk=z(2, 7, 2, 8), dv=z(2, 7, 2, 8))
    for bad in (dict(dq=z(2, 5, 2, 8)), dict(dk=z(2, 5, 2, 8)), dict(dout=z(2, 5, 4, 4)), dict(dtable=z(3, 4)), dict(table=table, bucket_of=of, dtable=z(4, 4)),
                dict(table=table, bucket_of=of, dtable=z(3, 4, dtype=torch.bfloat16)), dict(dv=z(2, 7, 2, 8, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            sf.attention_backward(**dict(back, **bad))
    if not torch.cuda.is_available():
        with pytest.raises(ValueError):                    # tensors of the host
            sf._on_current_device(q)


def test_blocks_refuse_what_kept_probabilities_cannot_do():
    """Lengths or a bias that a block would pass over."""
    from paper_2305_18513_amd import autograd as ag

    x, lengths = torch.zeros(1, 4, 64), torch.ones(1, dtype=torch.int32)
    p = ag.encoder_block_params(64, "cpu")
    for wrapped, recompute in ((True, False), (False, False), (False, True)):
        with pytest.raises(ValueError, match="go with recompute"):
            ag.frozen_encoder_block(x, p, 2, wrapped, recompute=recompute, lengths=lengths)
    p = ag.decoder_block_params(64, 2, 1, 64, "cpu")
    with pytest.raises(ValueError, match="go with recompute"):
        ag.decoder_block(x, p, 2, 1, torch.zeros(4, 32), lengths=lengths)
    with pytest.raises(ValueError, match="go with recompute"):
        ag.decoder_block(x, p, 2, 1, torch.zeros(4, 32), bias_table=torch.zeros(3, 2), bucket_of=torch.zeros(7, dtype=torch.int32))
