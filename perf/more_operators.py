"""What a fine-tuning step needs around its cached activations, each operator in its plain form and as the library's calls:
attention in one pass over the keys and its backward pass from recomputed probabilities, a learned position bias by buckets of
distance with its gradient, and AdamW over all tensors of a model at once, its states in 32 or 8 bits, with the layers' distances.

Sizes: 1 to 4097 queries and keys, heads of 32 to 128 elements, models of 0.4 to 150 million weights, fp32 and bf16.  ``own``
chooses between the two forms; ``exact`` has the results in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ALIGN = 256                                # elements: where tensors begin in a model's storage
FLOOR = 1e-3                               # of |w| in a layer's distance


def listed():
    def attention(name, **more):
        return dict(dict(name=name, kind="attention", step=True, apart=False, causal=False, ragged=False, buckets=0, reach=0, dtype="bf16"), **more)

    return [
        # One new token for each of 16 sequences over caches of unlike length, keys shared by four heads: bandwidth and launches count.
        attention("attn_token_bf16", step=False, batch=16, q_tokens=1, k_tokens=4096, q_heads=32, kv_heads=8, dim=128, ragged=True),
        # A prompt of odd length, heads as the rotation leaves them, nothing kept for a backward pass.
        attention("attn_prompt_bf16", step=False, batch=1, q_tokens=4097, k_tokens=4097, q_heads=24, kv_heads=8, dim=96, apart=True, causal=True),
        # A training step of an encoder's small padded batch, where launches count ...
        attention("attn_step_small_bf16", batch=8, q_tokens=128, k_tokens=128, q_heads=12, kv_heads=12, dim=64, ragged=True),
        # ... of a decoder of 16 heads of 64 (the large workloads' attention), ...
        attention("attn_step_bf16", batch=16, q_tokens=1024, k_tokens=1024, q_heads=16, kv_heads=16, dim=64, causal=True),
        # ... with keys shared by four heads, the largest batch, ...
        attention("attn_step_shared_bf16", batch=8, q_tokens=2048, k_tokens=2048, q_heads=32, kv_heads=8, dim=128, apart=True, causal=True),
        # ... and in fp32 of 37 images of 197 tokens.
        attention("attn_step_f32", batch=37, q_tokens=197, k_tokens=197, q_heads=12, kv_heads=12, dim=64, dtype="f32"),
        # Position bias: an encoder's padded batch, both directions ...
        attention("bias_step_bf16", batch=16, q_tokens=512, k_tokens=512, q_heads=12, kv_heads=12, dim=64, ragged=True, buckets=32, reach=128),
        # ... and a decoder's in fp32, of odd length, earlier keys alone.
        attention("bias_step_f32", batch=5, q_tokens=301, k_tokens=301, q_heads=8, kv_heads=8, dim=32, causal=True, buckets=20, reach=64, dtype="f32"),
        # AdamW: a tiny model, where launches count, ...
        dict(name="adamw_small_f32", kind="adamw", hidden=128, blocks=2, classes=2, dtype="f32", bits=32, block=0, frozen=0.0),
        # ... a base model in fp32 with a third of the layers frozen, ...
        dict(name="adamw_frozen_f32", kind="adamw", hidden=768, blocks=12, classes=3, dtype="f32", bits=32, block=0, frozen=0.34),
        # ... a large one in bf16 with its states in 8 bits, ...
        dict(name="adamw_8bit_bf16", kind="adamw", hidden=1024, blocks=12, classes=1000, dtype="bf16", bits=8, block=256, frozen=0.0),
        # ... and odd sizes in fp32 with states in 8 bits.
        dict(name="adamw_8bit_odd_f32", kind="adamw", hidden=509, blocks=3, classes=1003, dtype="f32", bits=8, block=64, frozen=0.2),
    ]


MOST_PAIRS = 8 * 32 * 2048 * 2048 * 128 // 2      # multiplications of the largest listed case, and its weights
MOST_WEIGHTS = 12 * 12 * 1024 * 1024


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if rng.random() < 0.3:
        hidden = _log_int(rng, 64, 1024)
        bits = rng.choice([32, 8])
        return dict(kind="adamw", hidden=hidden, blocks=_log_int(rng, 1, max(1, min(24, MOST_WEIGHTS // (12 * hidden * hidden)))),
                    classes=_log_int(rng, 2, 1003), dtype=dtype, bits=bits, block=rng.choice([32, 64, 128, 256]) if bits == 8 else 0,
                    frozen=rng.choice([0.0, 0.0, 0.2, 0.5]))
    dim = rng.choice([32, 40, 64, 64, 80, 96, 128])
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    q = kv * rng.choice([1, 1, 2, 4, 7] if kv <= 4 else [1, 2])
    step = rng.random() < 0.7
    k_tokens = _log_int(rng, 8 if step else 1, 4097)       # (a query that sees one key has gradients of rounding errors alone)
    q_tokens = 1 if not step and rng.random() < 0.5 else rng.choice([k_tokens, k_tokens, k_tokens, _log_int(rng, 1, 4097)])
    most = MOST_PAIRS // (q * q_tokens * k_tokens * dim * (4 if dtype == "f32" else 1))
    if most < 1:                           # one sequence of fewer heads
        q = kv = max(1, MOST_PAIRS // (q_tokens * k_tokens * dim * 4))
        kv = q = min(q, 4)
    buckets = rng.choice([0, 0, 2, 20, 32, 64])
    return dict(kind="attention", step=step, batch=_log_int(rng, 1, max(1, min(64, most))), q_tokens=q_tokens, k_tokens=k_tokens, q_heads=q, kv_heads=kv,
                dim=dim, apart=rng.random() < 0.3, causal=rng.random() < 0.5, ragged=rng.random() < 0.4, buckets=buckets,
                reach=rng.choice([32, 128, 500]) if buckets else 0, dtype=dtype)


# ------------------------------------------------------------------------------------------------------- inputs

def _activation(g, *shape):
    """N(0, 1) with one element in a thousand five times as large."""
    x = torch.randn(*shape, generator=g, device=DEV)
    hit = torch.randint(0, 1000, shape, generator=g, device=DEV, dtype=torch.int16) == 0
    return torch.where(hit, x * 5.0, x)


def _buckets_of(case):
    """The bucket of each distance, key minus query, from 1 - q_tokens on: half of a side's buckets hold one distance each, the others
    grow with its logarithm up to ``reach``; keys after the query have buckets of their own unless they are masked."""
    n, reach = case["buckets"], case["reach"]
    far = torch.arange(1 - case["q_tokens"], case["k_tokens"], dtype=torch.float64)
    side = n if case["causal"] else n // 2
    one = max(1, side // 2)
    away = torch.clamp(-far, min=0) if case["causal"] else far.abs()
    grown = one + torch.log(torch.clamp(away, min=1) / one) / math.log(max(reach, one + 1) / one) * (side - one)
    bucket = torch.where(away < one, away, torch.clamp(grown.floor(), min=one)).clamp(max=side - 1)
    if not case["causal"]:
        bucket = bucket + torch.where(far > 0, side, 0)
    return bucket.to(torch.int32).to(DEV)


def _model_sizes(case):
    """The tensors' element counts: for each block QKV, projection, two feed-forward matrices, two LayerNorms; then the classes."""
    H = case["hidden"]
    return [3 * H * H, H * H, 4 * H * H, 4 * H * H, H, H, H, H] * case["blocks"] + [case["classes"] * H, case["classes"]]


def _kept_v(v, block, dither):
    """(code, power of two) that a cache of v holds: 5 exponent and 3 fraction bits over a power of two for each run, rounded up where
    the dither (20 bits) carries; the smallest code but 0 for what is smaller than it."""
    word = v.view(torch.int32)
    top = (v.view(-1, block).amax(1).view(torch.int32) >> 23) - 30
    top = torch.clamp(top, min=1)[:, None]
    code = ((word + dither) >> 20).view(-1, block) - 8 * top
    code = torch.where(v.view(-1, block) > 0, code.clamp(1, 255), 0)
    return code, (top << 23).to(torch.int32).view(torch.float32)


def _kept_m(m, block):
    """(e4m3 values, scale) of runs: multiplied by 448 / max|m| and rounded to even; a run of zeros is kept as zeros."""
    runs = m.view(-1, block)
    top = runs.abs().amax(1, keepdim=True)
    whole = torch.full_like(top, 448.0)
    factor = whole / top
    fine = torch.isfinite(factor)
    return (runs * torch.where(fine, factor, 0.0)).to(torch.float8_e4m3fn), torch.where(fine, top / whole, 0.0)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    s = dict(case=case)
    if case["kind"] == "attention":
        B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "dim"))
        q, k, v = _activation(g, B, Tq, Hq, D).to(dtype), _activation(g, B, Tk, Hk, D).to(dtype), _activation(g, B, Tk, Hk, D).to(dtype)
        if case["apart"]:                  # as the heads' rotation leaves them
            s["q"], s["k"], s["v"] = q.transpose(1, 2).contiguous(), k.permute(0, 2, 3, 1).contiguous(), v.transpose(1, 2).contiguous()
        elif Tq == Tk:                     # the rows of one projection
            rows = torch.cat((q, k, v), 2).contiguous()
            s["q"], s["k"], s["v"] = rows[:, :, :Hq], rows[:, :, Hq : Hq + Hk], rows[:, :, Hq + Hk :]
        else:
            rows = torch.cat((k, v), 2).contiguous()
            s["q"], s["k"], s["v"] = q, rows[:, :, :Hk], rows[:, :, Hk:]
        s["lengths"] = None
        if case["ragged"]:                 # some sequence may have no key at all
            s["lengths"] = torch.randint(0 if B > 4 else Tk // 2, Tk + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
        s["table"] = s["bucket_of"] = None
        if case["buckets"]:
            s["table"] = torch.randn(case["buckets"], Hq, generator=g, device=DEV).to(dtype)
            s["bucket_of"] = _buckets_of(case)
        s["scale"] = 1.0 / math.sqrt(D)
        s["out"] = torch.empty(B, Tq, Hq, D, dtype=dtype, device=DEV)
        s["stats"] = torch.empty(B, Hq, Tq, 2, device=DEV)
        if case["step"]:
            s["dout"] = (torch.randn(B, Tq, Hq, D, generator=g, device=DEV) * 0.1).to(dtype)
            if case["apart"]:
                s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[n]) for n in "qkv")
            elif Tq == Tk:
                drows = torch.empty_like(rows)
                s["dq"], s["dk"], s["dv"] = drows[:, :, :Hq], drows[:, :, Hq : Hq + Hk], drows[:, :, Hq + Hk :]
            else:
                drows = torch.empty_like(rows)
                s["dq"], s["dk"], s["dv"] = torch.empty_like(q), drows[:, :, :Hk], drows[:, :, Hk:]
            s["dtable"] = torch.empty_like(s["table"]) if case["buckets"] else None
        return s
    # a model in the middle of its training: one storage, tensors that begin at multiples of ALIGN, zeros between them
    sizes = _model_sizes(case)
    spans = [-(-n // ALIGN) * ALIGN for n in sizes]
    starts = [sum(spans[:i]) for i in range(len(spans))]
    total, block = sum(spans), case["block"]
    s["sizes"], s["spans"] = torch.tensor(sizes, device=DEV), torch.tensor(spans, device=DEV)
    inside = (torch.arange(total, device=DEV) - torch.repeat_interleave(torch.tensor(starts, device=DEV), s["spans"])) < torch.repeat_interleave(s["sizes"], s["spans"])
    s["w"] = (torch.randn(total, generator=g, device=DEV) * 0.03 * inside).to(dtype)
    spread = 1e-3 * torch.exp(1.5 * torch.randn(total, generator=g, device=DEV))          # of each weight's gradients
    s["grad"] = (torch.randn(total, generator=g, device=DEV) * spread * inside).to(dtype)
    m = torch.randn(total, generator=g, device=DEV) * spread * 0.3 * inside
    v = spread.square() * torch.exp(0.3 * torch.randn(total, generator=g, device=DEV)) * inside
    if case["bits"] == 32:
        s["m"], s["v"], s["m_scales"], s["v_scales"] = m, v, None, None
    else:
        code, scale = _kept_m(m, block)
        s["m"], s["m_scales"] = code.view(torch.uint8).view(-1), scale.view(-1)
        code, scale = _kept_v(v, block, 1 << 19)
        s["v"], s["v_scales"] = code.to(torch.uint8).view(-1), scale.view(-1)
        s["m_read"], s["v_read"] = torch.empty(total, device=DEV), torch.empty(total, device=DEV)
    decay = [0.01 if n > case["hidden"] and n != case["classes"] else 0.0 for n in sizes]
    s["decay"] = torch.tensor(decay, device=DEV)
    s["frozen"] = (torch.rand(len(sizes), generator=g, device=DEV) < case["frozen"]).to(torch.uint8)
    s["distances"] = torch.empty(len(sizes), device=DEV)
    s.update(lr=2e-4, beta1=0.9, beta2=0.999, eps=1e-8, step=100 + seed % 1000, seed=seed % (1 << 31), factor=0.5)
    if own:
        from paper_2305_18513_amd import binding as sf

        def parts(t, per=1):
            return None if t is None else [t[a // per : a // per + -(-n // per)] for a, n in zip(starts, sizes)]

        s["numel"] = sizes
        s["workspace"] = torch.empty(sf.adamw_workspace(sizes), dtype=torch.uint8, device=DEV)
        sf.adamw_plan(parts(s["w"]), parts(s["grad"]), parts(s["m"]), parts(s["v"]), parts(s["m_scales"], block or 1), parts(s["v_scales"], block or 1),
                      decay, case["bits"], block, s["workspace"])
    return s


# -------------------------------------------------------------------------------------------------- plain forms

def _by_heads(s):
    """q (B, kv heads, group * q_tokens, D), k and v (B, kv heads, k_tokens, D) in 32 bits."""
    case = s["case"]
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "dim"))
    if case["apart"]:
        q, k, v = s["q"].float(), s["k"].float().transpose(2, 3).contiguous(), s["v"].float()
    else:
        q, k, v = (s[n].float().transpose(1, 2).contiguous() for n in "qkv")
    return q.reshape(B, Hk, Hq // Hk * Tq, D), k, v


def _unseen(s):
    """Which pairs are masked, (B or 1, 1, q_tokens, k_tokens), or None."""
    case = s["case"]
    Tq, Tk = case["q_tokens"], case["k_tokens"]
    key = torch.arange(Tk, device=DEV)
    hidden = None
    if case["causal"]:
        hidden = (key[None, :] > torch.arange(Tq, device=DEV)[:, None] + (Tk - Tq))[None, None]
    if s["lengths"] is not None:
        past = (key[None, :] >= s["lengths"][:, None])[:, None, None, :]
        hidden = past if hidden is None else hidden | past
    return hidden


def _plain_attention(s):
    case = s["case"]
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "dim"))
    dtype, shared = s["out"].dtype, (B, Hk, Hq // Hk * Tq, Tk)
    q, k, v = _by_heads(s)
    x = torch.matmul(q, k.transpose(2, 3)).view(B, Hq, Tq, Tk).mul_(s["scale"])
    if case["buckets"]:
        at = torch.arange(Tk, device=DEV)[None, :] - torch.arange(Tq, device=DEV)[:, None] + (Tq - 1)
        bucket = s["bucket_of"].long()[at]
        x += s["table"].float().t()[:, bucket]
    hidden = _unseen(s)
    if hidden is not None:
        x.masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(torch.where(torch.isinf(top), 0.0, top)))
    total = p.sum(-1, keepdim=True)
    p *= torch.where(total > 0, 1.0 / total, 0.0)
    o = torch.matmul(p.view(shared), v).view(B, Hq, Tq, D)
    out = dict(out=o.transpose(1, 2).to(dtype).contiguous(), stats=torch.cat((top, total), -1))
    if not case["step"]:
        return out
    do = s["dout"].float().transpose(1, 2).contiguous()
    dp = torch.matmul(do.view(B, Hk, -1, D), v.transpose(2, 3)).view(B, Hq, Tq, Tk)
    dv = torch.matmul(p.view(shared).transpose(2, 3), do.view(B, Hk, -1, D))
    ds = dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    if case["buckets"]:
        # rows last to first, each a place further right: the columns are the distances
        by_distance = torch.nn.functional.pad(ds.sum(0).flip(1), (0, Tq)).view(Hq, -1)[:, : Tq * (Tq + Tk - 1)].view(Hq, Tq, -1).sum(1, dtype=torch.float64)
        out["dtable"] = torch.zeros(case["buckets"], Hq, dtype=torch.float64, device=DEV).index_add_(0, s["bucket_of"], by_distance.t().contiguous()).to(dtype)
    ds *= s["scale"]
    dq, dk = torch.matmul(ds.view(shared), k).view(B, Hq, Tq, D), torch.matmul(ds.view(shared).transpose(2, 3), q)
    if case["apart"]:
        return dict(out, dq=dq.to(dtype), dk=dk.transpose(2, 3).to(dtype).contiguous(), dv=dv.to(dtype))
    return dict(out, dq=dq.transpose(1, 2).to(dtype), dk=dk.transpose(1, 2).to(dtype), dv=dv.transpose(1, 2).to(dtype))


def _mix(x):
    """32 bits from 32 bits, in int64."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _dither(s):
    """20 bits for each weight: by fours of a tensor's weights one word, turned by 8 bits for each of the four."""
    layer = torch.arange(len(s["sizes"]), device=DEV)
    key = _mix(s["seed"] ^ _mix(s["step"] ^ _mix(layer + 1)))
    ends = torch.cumsum(s["spans"], 0)
    place = torch.arange(s["w"].numel(), device=DEV) - torch.repeat_interleave(ends - s["spans"], s["spans"])
    word = _mix((torch.repeat_interleave(key, s["spans"]) + (place >> 2)) & 0xFFFFFFFF)
    turn = 8 * (place & 3)
    return ((((word << turn) | (word >> (32 - turn))) & 0xFFFFFFFF) >> 12).to(torch.int32)


def _read_m(s):
    return (s["m"].view(torch.float8_e4m3fn).float().view(-1, s["case"]["block"]) * s["m_scales"][:, None]).view(-1)


def _read_v(s):
    code = s["v"].to(torch.int32).view(-1, s["case"]["block"])
    return torch.where(code > 0, (s["v_scales"].view(torch.int32)[:, None] + (code << 20)).view(torch.float32), 0.0).view(-1)


def _new_states(s, m, v):
    """Both moments, in 32 bits as they are defined: products rounded, then their sum."""
    g = s["grad"].float() * s["factor"]
    return m * s["beta1"] + g * (1.0 - s["beta1"]), v * s["beta2"] + (g * (1.0 - s["beta2"])) * g


def _plain_adamw(s):
    case = s["case"]
    w = s["w"].float()
    if case["bits"] == 8:
        m, v = _new_states(s, _read_m(s), _read_v(s))
    else:
        m, v = _new_states(s, s["m"], s["v"])
    each = torch.repeat_interleave(torch.stack((s["decay"], s["frozen"].float())), s["spans"], 1)
    rate = s["lr"] / (1.0 - s["beta1"] ** s["step"])
    delta = -(w * (s["lr"] * each[0]) + m / (torch.sqrt(v) * (1.0 / math.sqrt(1.0 - s["beta2"] ** s["step"])) + s["eps"]) * rate)
    live = each[1] == 0
    delta = torch.where(live, delta, 0.0)
    terms = (delta.abs() / w.abs().clamp(min=FLOOR)).double().view(-1, ALIGN).sum(1)
    s["distances"].copy_(torch.zeros(len(s["sizes"]), dtype=torch.float64, device=DEV).index_add_(
        0, torch.repeat_interleave(torch.arange(len(s["sizes"]), device=DEV), s["spans"] // ALIGN), terms) / s["sizes"])
    s["w"].copy_(w + delta)
    if case["bits"] == 32:
        s["m"].copy_(torch.where(live, m, s["m"]))
        s["v"].copy_(torch.where(live, v, s["v"]))
        return dict(w=s["w"], m=s["m"], v=s["v"], distances=s["distances"])
    run = live.view(-1, case["block"])
    for name, (code, scale) in (("m", _kept_m(m, case["block"])), ("v", _kept_v(v, case["block"], _dither(s)))):
        byte = code.view(torch.uint8) if name == "m" else code.to(torch.uint8)
        s[name].copy_(torch.where(run, byte, s[name].view(run.shape)).view(-1))
        s[name + "_scales"].copy_(torch.where(run[:, 0], scale[:, 0], s[name + "_scales"]))
    return dict(w=s["w"], m=_read_m(s), v=_read_v(s), distances=s["distances"])


# ------------------------------------------------------------------------------------------------------ one pass

def _own_attention(s):
    from paper_2305_18513_amd import binding as sf
    case = s["case"]
    layout = sf.HEADS_APART if case["apart"] else sf.HEADS_ROWS
    sf.attention_forward(s["q"], s["k"], s["v"], layout, s["scale"], case["causal"], s["lengths"], s["table"], s["bucket_of"], s["out"], s["stats"])
    out = dict(out=s["out"], stats=s["stats"])
    if case["step"]:
        sf.attention_backward(s["dout"], s["q"], s["k"], s["v"], layout, s["scale"], case["causal"], s["lengths"], s["table"], s["bucket_of"], s["out"],
                              s["stats"], s["dq"], s["dk"], s["dv"], s["dtable"])
        out.update(dq=s["dq"], dk=s["dk"], dv=s["dv"])
        if case["buckets"]:
            out["dtable"] = s["dtable"]
    return out


def _own_adamw(s):
    from paper_2305_18513_amd import binding as sf
    case = s["case"]
    dt = sf.F32 if case["dtype"] == "f32" else sf.BF16
    sf.adamw_run(s["numel"], dt, dt, case["bits"], case["block"], s["lr"], s["beta1"], s["beta2"], s["eps"], s["step"], s["workspace"],
                 grad_factor=s["factor"], seed=s["seed"], frozen=s["frozen"], floor=FLOOR, d_out=s["distances"])
    if case["bits"] == 32:
        return dict(w=s["w"], m=s["m"], v=s["v"], distances=s["distances"])
    sf.adamw_states(s["m"], s["m_scales"], s["v"], s["v_scales"], case["block"], s["m_read"], s["v_read"])
    return dict(w=s["w"], m=s["m_read"], v=s["v_read"], distances=s["distances"])


def run(s):
    if s["case"]["kind"] == "attention":
        return _own_attention(s) if own else _plain_attention(s)
    return _own_adamw(s) if own else _plain_adamw(s)


def _pairs(case):
    """How many keys all queries of a head see together, where no sequence is shorter."""
    Tq, Tk = case["q_tokens"], case["k_tokens"]
    if not case["causal"]:
        return Tq * Tk
    first = max(0, Tq - Tk)                # queries before it see none
    low = max(0, Tk - Tq) + 1
    return (low + Tk) * (Tq - first) // 2


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "attention":
        B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "dim"))
        rows, keys = B * Tq * Hq * D * e, B * Tk * Hk * D * e * (0.5 if case["ragged"] and B > 4 else 0.75 if case["ragged"] else 1.0)
        pairs = B * Hq * D * _pairs(case) * (0.5 if case["ragged"] and B > 4 else 0.75 if case["ragged"] else 1.0)
        moved = 2 * rows + 2 * keys + 8 * B * Hq * Tq
        if case["step"]:
            moved += 4 * rows + 2 * keys + 2 * B * Tk * Hk * D * e + 8 * B * Hq * Tq
        return dict(bytes=moved, flops=(14 if case["step"] else 4) * pairs)
    n, live = sum(_model_sizes(case)), 1.0 - case["frozen"]
    held = 16 if case["bits"] == 32 else 4 + 16 / case["block"]
    moved = n * live * (3 * e + held)
    if case["bits"] == 8:
        moved += n * (2 + 8 / case["block"] + 8)
    return dict(bytes=moved, flops=20 * n * live)


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_attention(case, s):
    B, Tq, Tk, Hq, Hk, D = (case[k] for k in ("batch", "q_tokens", "k_tokens", "q_heads", "kv_heads", "dim"))
    group = Hq // Hk
    every = {}
    for b in range(B):                     # a sequence at a time: (heads, tokens, D)
        q, k, v = (s[n][b] for n in "qkv")
        if case["apart"]:
            k = k.permute(0, 2, 1)
        else:
            q, k, v = (t.permute(1, 0, 2) for t in (q, k, v))
        q, k, v = q.double(), k.double().repeat_interleave(group, 0), v.double().repeat_interleave(group, 0)
        x = q @ k.mT * s["scale"]
        i, j = torch.arange(Tq, device=DEV)[:, None], torch.arange(Tk, device=DEV)[None, :]
        if case["buckets"]:
            bucket = s["bucket_of"][(j - i + Tq - 1).view(-1)].long()
            x = x + s["table"].double()[bucket].t().reshape(Hq, Tq, Tk)
        seen = torch.ones(Tq, Tk, dtype=torch.bool, device=DEV)
        if case["causal"]:
            seen = seen & (j - i <= Tk - Tq)
        if s["lengths"] is not None:
            seen = seen & (j < s["lengths"][b])
        x = torch.where(seen, x, -math.inf)
        top = x.max(-1).values if Tk else x.new_full((Hq, Tq), -math.inf)
        total = torch.exp(x - torch.nan_to_num(top, neginf=0.0)[..., None]).sum(-1)
        p = torch.softmax(x, -1).nan_to_num(0.0)
        o = p @ v
        got = dict(out=o.permute(1, 0, 2), stats=torch.stack((top, total), -1))
        if case["step"]:
            do = s["dout"][b].double().permute(1, 0, 2)
            ds = p * (do @ v.mT - (do * o).sum(-1)[..., None])
            dq, dk, dv = ds @ k * s["scale"], ds.mT @ q * s["scale"], p.mT @ do
            dk, dv = (t.view(Hk, group, Tk, D).sum(1) for t in (dk, dv))
            got.update(dq=dq, dk=dk, dv=dv)
            if case["apart"]:
                got["dk"] = dk.permute(0, 2, 1)
            else:
                got.update({n: got[n].permute(1, 0, 2) for n in ("dq", "dk", "dv")})
            if case["buckets"]:
                got["dtable"] = torch.zeros(case["buckets"], Hq, dtype=torch.float64, device=DEV).index_add_(0, bucket, ds.view(Hq, -1).t().contiguous())
        for name, t in got.items():
            every.setdefault(name, []).append(t)
    return {name: sum(ts) if name == "dtable" else torch.stack(ts) for name, ts in every.items()}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    spans, block = s["spans"], case["block"]
    tensor = torch.repeat_interleave(torch.arange(len(spans), device=DEV), spans)
    live = s["frozen"][tensor] == 0
    w, g = s["w"].double(), s["grad"].double() * s["factor"]
    m, v = (s["m"], s["v"]) if case["bits"] == 32 else (_read_m(s), _read_v(s))
    m64 = s["beta1"] * m.double() + (1 - s["beta1"]) * g
    v64 = s["beta2"] * v.double() + (1 - s["beta2"]) * g ** 2
    step = m64 / (1 - s["beta1"] ** s["step"]) / ((v64 / (1 - s["beta2"] ** s["step"])) ** 0.5 + s["eps"])
    delta = torch.where(live, -s["lr"] * (s["decay"].double()[tensor] * w + step), 0.0)
    ratio = delta.abs() / torch.maximum(w.abs(), torch.full_like(w, FLOOR))
    ends = torch.cumsum(spans, 0)
    summed = torch.cat((ratio.new_zeros(1), torch.cumsum(ratio, 0)))
    out = dict(w=w + delta, distances=(summed[ends] - summed[ends - spans]) / s["sizes"])
    if case["bits"] == 32:
        return dict(out, m=torch.where(live, m64, m.double()), v=torch.where(live, v64, v.double()))
    # what 8 bits hold: codes are whole numbers that 32-bit arithmetic defines, their values are formed in 64
    m32, v32 = _new_states(s, m, v)
    e4m3, scale = _kept_m(m32, block)
    code, power = _kept_v(v32, block, _dither(s))
    held_v = torch.where(code > 0, power.double() * torch.exp2((code // 8).double()) * (1 + (code % 8).double() / 8), 0.0)
    held_m = e4m3.double() * scale.double()
    return dict(out, m=torch.where(live, held_m.view(-1), m.double()), v=torch.where(live, held_v.view(-1), v.double()))
