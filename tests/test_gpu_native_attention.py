"""The native form of the attention and AdamW calls against the general (ctypes) path: the same bytes, exception or status over every
form of argument."""
import pytest
import torch

from paper_2305_18513_amd import binding as sf
from tests.gpu_util import require_gpu
from tests.test_gpu_native_binding import _general, _outcome, _Subclass, _variants

pytestmark = pytest.mark.gpu


def _calls(dt, layout):
    g = torch.Generator(device="cuda").manual_seed(3)
    B, Tq, Tk, Hq, Hk, D = 2, 20, 36, 4, 2, 16
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    if layout == sf.HEADS_ROWS:
        rows = rand(B, Tk, 2 * Hk, D)
        q, k, v = rand(B, Tq, Hq, D), rows[:, :, :Hk], rows[:, :, Hk:]
    else:
        q, k, v = rand(B, Hq, Tq, D), rand(B, Hk, D, Tk), rand(B, Hk, Tk, D)
    lengths = torch.tensor([30, 36], dtype=torch.int32, device="cuda")
    table, of = rand(5, Hq), sf.distance_buckets(Tq, Tk, 5, 20)
    out, stats, dout = rand(B, Tq, Hq, D), torch.empty(B, Hq, Tq, 2, device="cuda"), rand(B, Tq, Hq, D)
    forward = [q, k, v, layout, 0.25, True, lengths, table, of, out, stats]
    sf.attention_forward(*forward)
    new = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v)]
    backward = [dout, q, k, v, layout, 0.25, True, lengths, table, of, out.clone(), stats.clone(), *new, torch.empty_like(table)]
    plain = [q, k, v, layout, 0.25, False, None, None, None, out, stats]
    numel = [300, 8]
    w, grad, m = ([rand(n) if i < 2 else torch.zeros(n, device="cuda") for n in numel] for i in range(3))
    vv = [torch.zeros(n, device="cuda") for n in numel]
    ws = torch.empty(sf.adamw_workspace(numel), dtype=torch.uint8, device="cuda")
    frozen = torch.tensor([1, 1], dtype=torch.uint8, device="cuda")       # the step itself changes its inputs: what is compared touches nothing
    sf.adamw_plan(w, grad, m, vv, None, None, [0.1, 0.0], 32, 0, ws)
    kind = sf.F32 if dt == torch.float32 else sf.BF16
    step = [numel, kind, kind, 32, 0, 1e-3, 0.9, 0.999, 1e-8, 3, ws, 1.0, 5, None, frozen, 0.0, torch.empty(2, device="cuda")]
    return {"attention_forward": (sf.attention_forward, forward, (9, 10)), "attention_forward_plain": (sf.attention_forward, plain, (9, 10)),
            "attention_backward": (sf.attention_backward, backward, (12, 13, 14, 15)), "adamw_run": (sf.adamw_run, step, (16,))}


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", [sf.HEADS_ROWS, sf.HEADS_APART])
@pytest.mark.parametrize("name", ["attention_forward", "attention_forward_plain", "attention_backward", "adamw_run"])
def test_both_paths_give_the_same(name, layout, dt):
    require_gpu()
    fn, args, outs = _calls(dt, layout)[name]
    outputs = [args[i] for i in outs]
    assert getattr(sf, "_native_" + fn.__name__)(*args, *([None] * (fn.__code__.co_argcount - len(args)))) is None     # taken
    assert _outcome(lambda: fn(*args), outputs) == _outcome(lambda: _general(fn, *args), outputs)
    stream = torch.cuda.current_stream().cuda_stream
    assert _outcome(lambda: fn(*args, stream=stream), outputs) == _outcome(lambda: _general(fn, *args, stream=stream), outputs)
    for i, a in enumerate(args):
        if name == "adamw_run" and i in (10, 14):          # workspaces without the plan, masks that let layers change
            continue
        for other in _variants(a):
            changed = list(args)
            changed[i] = other
            seen = [other if j == i else args[j] for j in outs] if isinstance(other, torch.Tensor) and other.is_cuda and i in outs else outputs
            seen = [t.detach() for t in seen if t.is_contiguous() and type(t) is not _Subclass]
            got, want = _outcome(lambda: fn(*changed), seen), _outcome(lambda: _general(fn, *changed), seen)
            assert got == want, "argument %d as %r" % (i, type(other))
