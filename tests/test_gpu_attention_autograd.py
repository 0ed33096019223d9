"""GPU: attention that forms its probabilities again, through torch.autograd, in the blocks, and with AdamW in a step as a fine-tuning
loop makes it."""
import pytest
import torch

from paper_2305_18513_amd import autograd as ag
from paper_2305_18513_amd import binding as sf
from tests.gpu_util import require_gpu
from tests.test_gpu_decoder import _plain_block

pytestmark = pytest.mark.gpu


def _inputs(dtype, B=2, T=70, Hq=4, Hk=2, D=64, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(B, T, (Hq + 2 * Hk) * D, generator=g, device="cuda").to(dtype)
    dout = torch.randn(B, T, Hq * D, generator=g, device="cuda").to(dtype)
    table, of = torch.randn(9, Hq, generator=g, device="cuda").to(dtype), sf.distance_buckets(T, T, 9, 30)
    return qkv, dout, table, of, torch.tensor([T, T // 2], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_functions_are_the_calls(dtype):
    """Rows, operands apart and the calls themselves give the same bits; what needs no gradient gets none."""
    require_gpu()
    qkv, dout, table, of, lengths = _inputs(dtype)
    B, T, Hq, Hk, D = 2, 70, 4, 2, 64
    q, k, v = qkv.view(B, T, Hq + 2 * Hk, D).split((Hq, Hk, Hk), 2)
    out, stats = torch.empty(B, T, Hq, D, dtype=dtype, device="cuda"), torch.empty(B, Hq, T, 2, device="cuda")
    args = (sf.HEADS_ROWS, 0.125, True, lengths, table, of)
    sf.attention_forward(q, k, v, *args, out, stats)
    want, dtable = torch.empty_like(qkv), torch.empty_like(table)
    sf.attention_backward(dout.view(B, T, Hq, D), q, k, v, *args, out, stats, *want.view(B, T, Hq + 2 * Hk, D).split((Hq, Hk, Hk), 2), dtable)

    rows, bias = qkv.clone().requires_grad_(True), table.clone().requires_grad_(True)
    y = ag.SelfAttentionFunction.apply(rows, Hq, Hk, 0.125, True, lengths, bias, of)
    assert torch.equal(y, out.view(B, T, -1))
    got = torch.autograd.grad(y, (rows, bias), dout)
    assert torch.equal(got[0], want) and torch.equal(got[1], dtable)

    apart = [t.clone().requires_grad_(True) for t in (q.transpose(1, 2), k.permute(0, 2, 3, 1), v.transpose(1, 2))]
    z = ag.AttentionFunction.apply(*apart, 0.125, True, lengths, bias, of, sf.HEADS_APART)
    assert torch.equal(z, out)
    dq, dkt, dv, db = torch.autograd.grad(z, (*apart, bias), dout.view(B, T, Hq, D).expand(B, T, Hq, D))
    assert torch.equal(torch.cat((dq.transpose(1, 2), dkt.permute(0, 3, 1, 2), dv.transpose(1, 2)), 2).reshape(B, T, -1), want) and torch.equal(db, dtable)

    frozen = ag.SelfAttentionFunction.apply(rows, Hq, Hk, 0.125, True, lengths, table, of)
    assert torch.equal(torch.autograd.grad(frozen, rows, dout)[0], want)
    only = ag.SelfAttentionFunction.apply(qkv, Hq, Hk, 0.125, True, lengths, bias, of)
    assert torch.equal(torch.autograd.grad(only, bias, dout)[0], dtable)


def test_nothing_is_kept_without_gradients_and_second_ones_are_refused():
    require_gpu()
    qkv, dout, table, of, lengths = _inputs(torch.float32)
    rows = qkv.clone().requires_grad_(True)
    with torch.no_grad():
        assert not ag.SelfAttentionFunction.apply(rows, 4, 2, 0.125, False, lengths, table, of).requires_grad
    y = ag.SelfAttentionFunction.apply(rows, 4, 2, 0.125, False, lengths, table, of)
    (d,) = torch.autograd.grad(y, rows, dout, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(d.sum(), rows)
    with pytest.raises((TypeError, ValueError)):
        ag.SelfAttentionFunction.apply(rows.half(), 4, 2, 0.125)
    with pytest.raises(sf.SlimfitError):                   # heads of 192
        ag.SelfAttentionFunction.apply(torch.randn(1, 8, 3 * 192, device="cuda"), 1, 1, 0.125)
    with pytest.raises(ValueError):
        ag.SelfAttentionFunction.apply(rows, 4, 2, 0.125, False, lengths, table.bfloat16(), of)
    with pytest.raises(ValueError):
        ag.SelfAttentionFunction.apply(rows.cpu(), 4, 2, 0.125)


def test_encoder_block():
    """Against the same block in plain torch: equal but for fp32 sums forward; gradients within the caches' errors (two norms that keep
    everything, GELU's input in 8 bits: 0.5 % of a block's values), and fewer bytes held than with kept probabilities."""
    require_gpu()
    B, T, H, heads = 4, 300, 256, 4
    p = ag.encoder_block_params(H, "cuda", 1)
    x = torch.randn(B, T, H, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda", requires_grad=True)
    args = (p, heads, True, 1000000, 8, 32)
    out, want = ag.frozen_encoder_block(x, *args, recompute=True), ag.frozen_encoder_block(x, p, heads, False)
    # six sums of up to 4 H terms one after the other
    assert float((out - want).abs().max().detach()) <= 6 * 4 * H * 2.0 ** -24 * float(want.abs().max().detach())
    dout = torch.randn_like(out)
    got, ref = torch.autograd.grad(out, x, dout)[0], torch.autograd.grad(want, x, dout)[0]
    assert float((got - ref).norm() / ref.norm()) <= 3 * 0.005
    del out, want, got, ref
    kept = [ag.held_activation_bytes(lambda: ag.frozen_encoder_block(x, *args, recompute=again))[0] for again in (True, False)]
    assert kept[0] < kept[1]
    # padding takes no part: the first tokens' results are those of the shorter batch
    lengths = torch.full((B,), 200, dtype=torch.int32, device="cuda")
    with torch.no_grad():
        padded, short = ag.frozen_encoder_block(x, *args, recompute=True, lengths=lengths), ag.frozen_encoder_block(x[:, :200].contiguous(), *args, recompute=True)
    assert float((padded[:, :200] - short).abs().max()) <= 6 * 4 * H * 2.0 ** -24 * float(short.abs().max())


@pytest.mark.parametrize("hidden,heads,kv_heads,T", [(256, 4, 2, 48), (128, 4, 1, 33), (128, 2, 2, 2100)])
def test_decoder_block(hidden, heads, kv_heads, T):
    """As with kept probabilities, and past their 2048 tokens, against plain torch in 64 bits."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(T)
    p = ag.decoder_block_params(hidden, heads, kv_heads, 2 * hidden, "cuda", 1)
    table = sf.rotary_table(T + 3, hidden // heads)
    x = torch.randn(2, T, hidden, generator=g, device="cuda", requires_grad=True)
    dout = torch.randn(2, T, hidden, generator=g, device="cuda")
    out = ag.decoder_block(x, p, heads, kv_heads, table, None, 1000000, 8, 32, recompute=True)
    wide = {n: t.detach().double().requires_grad_(True) for n, t in p.items()}
    xw = x.detach().double().requires_grad_(True)
    want = _plain_block(xw, wide, heads, kv_heads, table.double(), sf.ACT_SILU)
    # fp32 sums of up to max(2 * hidden, T) terms, six of them one after the other
    assert float((out.double() - want).abs().max().detach()) <= 6 * max(512, T) * 2.0 ** -24 * float(want.abs().max().detach())
    got = torch.autograd.grad(out, [x, *p.values()], dout)
    ref = torch.autograd.grad(want, [xw, *wide.values()], dout.double())
    for name, a, b in zip(["x", *p], got, ref):
        # caches of 8 bits are off by 0.5 % of their values: nine of them (two norms, the heads, four linear layers, the gate) added up
        assert float((a.double() - b).norm() / b.norm()) <= 9 * 0.005, name


def test_steps_of_a_fine_tuning_loop():
    """Two decoder blocks with a position bias, their gradients, AdamW over all of their tensors with the layers' distances, and the
    scheduler's choice of what the next step freezes: three steps, the weights against torch's AdamW on the same gradients."""
    require_gpu()
    hidden, heads, T = 128, 2, 90
    blocks = [ag.decoder_block_params(hidden, heads, 1, 256, "cuda", s) for s in (1, 2)]
    biases = [torch.nn.Parameter(torch.zeros(16, heads, device="cuda")) for _ in blocks]
    params = [t for p, b in zip(blocks, biases) for t in (*p.values(), b)]
    table, of = sf.rotary_table(T, hidden // heads), sf.distance_buckets(T, T, 16, 50, False)
    lengths = torch.tensor([T, 60], dtype=torch.int32, device="cuda")
    x = torch.randn(2, T, hidden, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    numel = [t.numel() for t in params]
    L = len(params)
    for t in params:
        t.grad = torch.zeros_like(t)
    m, v = ([torch.zeros_like(t) for t in params] for _ in range(2))
    decay = [0.01 if t.dim() == 2 else 0.0 for t in params]
    ws, d = torch.empty(sf.adamw_workspace(numel), dtype=torch.uint8, device="cuda"), torch.empty(L, device="cuda")
    data = [t.data for t in params]
    sf.adamw_plan(data, [t.grad for t in params], m, v, None, None, decay, 32, 0, ws)
    mirror = [t.detach().clone().requires_grad_(True) for t in params]
    other = torch.optim.AdamW([dict(params=[t], weight_decay=w) for t, w in zip(mirror, decay)], lr=1e-3, eps=1e-8, foreach=False)
    apart = [0.0] * L
    distances, mask = torch.zeros(L).numpy(), torch.zeros(L, dtype=torch.uint8)
    for step in (1, 2, 3):
        for t, f in zip(params, mask.tolist()):
            t.requires_grad_(not f)
            t.grad.zero_()
        y = x
        for p, b in zip(blocks, biases):
            y = ag.decoder_block(y, p, heads, 1, table, None, 1000000, 8, 32, recompute=True, lengths=lengths, bias_table=b, bucket_of=of)
        (y.square().mean() * 100).backward()
        del y
        before = [t.detach().clone() for t in params]
        for t, o, f in zip(params, mirror, mask.tolist()):
            o.grad = None if f else t.grad.detach().clone()
        sf.adamw_run(numel, sf.F32, sf.F32, 32, 0, 1e-3, 0.9, 0.999, 1e-8, step, ws, frozen=mask.cuda(), floor=1e-3, d_out=d)
        # torch's optimizer counts a parameter's own steps, frozen ones are behind: so does its correction, which is set here
        for o in mirror:
            if o in other.state and o.grad is not None:
                other.state[o]["step"].fill_(step - 1)
        other.step()
        for i, (t, o, w) in enumerate(zip(params, mirror, before)):
            if mask[i]:
                assert torch.equal(t, w) and float(d[i]) == 0.0
                continue
            moved = (t.detach().double() - w.double()).abs()
            # Either form of the step is within twenty roundings of the move and two of the weight.  The two begin a step where they ended
            # the last: w' = (1 - lr * decay) w - move keeps what they were apart, so a step's bound comes on top of those before it.
            apart[i] = apart[i] + 40 * 2.0 ** -24 * (moved + 1e-3) + 4 * 2.0 ** -24 * w.double().abs()
            assert bool(((t.detach().double() - o.detach().double()).abs() <= apart[i]).all()), (step, i)
            want = (moved / w.double().abs().clamp(min=1e-3)).mean()
            # the weights' own rounding is in `moved`, not in the distance: 2^-24 of a weight over it, or over the floor
            assert abs(float(d[i]) - float(want)) <= 2.0 ** -22 + 1e-5 * float(want)
            assert bool(moved.any()), i
        if step == 1:                                      # first steps of a fresh layer have no state in torch's
            assert all(len(other.state[o]) for o in mirror)
        sf.ils_update(distances, d.cpu().numpy(), mask.numpy())
        _, chosen = sf.ils_select(distances, sf.freeze_count(L, 0.3))
        mask = torch.from_numpy(chosen.copy())
    assert int(mask.sum()) == int(L * 0.3)


def test_a_captured_step_replays_to_the_eager_gradients():
    require_gpu()
    qkv, dout, table, of, lengths = _inputs(torch.bfloat16)
    rows, bias = qkv.clone().requires_grad_(True), table.clone().requires_grad_(True)

    def step():
        y = ag.SelfAttentionFunction.apply(rows, 4, 2, 0.125, True, lengths, bias, of)
        return (y, *torch.autograd.grad(y, (rows, bias), dout))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = step()
    torch.cuda.synchronize()
    del warm
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for seed in (1, 2, 3):
        new = _inputs(torch.bfloat16, seed=seed)
        with torch.no_grad():
            rows.copy_(new[0])
            dout.copy_(new[1])
            bias.copy_(new[2])
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, [t.detach().clone() for t in step()]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("B,T", [(0, 5), (2, 0), (0, 0)])
def test_no_sequences_and_no_tokens(B, T):
    """A batch that is empty, or whose sequences are: empty results and gradients, and a table's that is 0."""
    require_gpu()
    Hq, Hk, D = 4, 2, 16
    table = torch.randn(3, Hq, device="cuda", requires_grad=True)
    of = torch.zeros(max(0, 2 * T - 1), dtype=torch.int32, device="cuda")
    rows = torch.randn(B, T, (Hq + 2 * Hk) * D, device="cuda", requires_grad=True)
    y = ag.SelfAttentionFunction.apply(rows, Hq, Hk, 0.25, True, None, table, of)
    assert y.shape == (B, T, Hq * D)
    drows, dtable = torch.autograd.grad(y.sum(), (rows, table))
    assert drows.shape == rows.shape and bool((dtable == 0).all())
    q, k, v = (torch.randn(B, T, h, D, device="cuda", requires_grad=True) for h in (Hq, Hk, Hk))
    y = ag.AttentionFunction.apply(q, k, v, 0.25, True, None, table, of)
    assert y.shape == (B, T, Hq, D)
    *grads, dtable = torch.autograd.grad(y.sum(), (q, k, v, table))
    assert all(g.shape == t.shape for g, t in zip(grads, (q, k, v))) and bool((dtable == 0).all())
