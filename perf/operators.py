"""The operators around a decoder layer's activations that are kept in 8 or 4 bits, each in its plain form and as the
library's calls: the queries' and keys' norm and position rotation on the way out of the projection's rows (with the
cache of what their backward pass reads), gated activations around the cache of their input, and the weight gradient of a
linear layer straight from the cache of its input.

Sizes: hidden 128 to 4096, 1 to 16384 tokens in a batch, fp32 and bf16, caches of 8 and 4 bits with a scale for each 32 to
256 elements.  ``own`` chooses between the two forms; ``exact`` has the results in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
ROTARY_BASE = 10000.0


def listed():
    return [
        # One new token for each of 64 sequences at unlike positions, on its way to attention: launches are what counts.
        dict(name="heads_tokens_bf16", kind="heads", step=False, batch=64, tokens=1, q_heads=32, kv_heads=8, dim=128, rotary=128,
             adjacent=False, norm=True, ids="far", dtype="bf16", bits=0, block=0),
        # A prompt of odd length, nothing kept, heads of 96 elements of which half turn.
        dict(name="heads_prompt_bf16", kind="heads", step=False, batch=1, tokens=4097, q_heads=24, kv_heads=8, dim=96, rotary=48,
             adjacent=False, norm=True, ids="none", dtype="bf16", bits=0, block=0),
        # A training step's forward and backward pass: 16 heads of 64 (the large workloads' attention), keys not shared ...
        dict(name="heads_step_bf16", kind="heads", step=True, batch=16, tokens=1024, q_heads=16, kv_heads=16, dim=64, rotary=64,
             adjacent=False, norm=True, ids="none", dtype="bf16", bits=8, block=64),
        # ... keys shared by four heads each, the largest batch ...
        dict(name="heads_step_shared_bf16", kind="heads", step=True, batch=8, tokens=2048, q_heads=32, kv_heads=8, dim=128, rotary=128,
             adjacent=False, norm=True, ids="none", dtype="bf16", bits=8, block=128),
        # ... and in fp32 the last, partial batch of 197 tokens, neighbours turned, positions with padding, 4 bits.
        dict(name="heads_step_f32", kind="heads", step=True, batch=37, tokens=197, q_heads=12, kv_heads=12, dim=64, rotary=32,
             adjacent=True, norm=True, ids="padded", dtype="f32", bits=4, block=32),
        # A gated feed-forward's activation for one token, nothing kept.
        dict(name="gated_token_bf16", kind="gated", step=False, rows=1, width=4096, act="silu", dtype="bf16", bits=0, block=0),
        # Its training step: a small ragged batch, ...
        dict(name="gated_step_small_bf16", kind="gated", step=True, rows=513, width=1408, act="silu", dtype="bf16", bits=8, block=128),
        # ... the partial batch of 197 tokens in fp32 and 4 bits, ...
        dict(name="gated_step_f32", kind="gated", step=True, rows=7289, width=2048, act="gelu", dtype="f32", bits=4, block=64),
        # ... and the largest batch.
        dict(name="gated_step_bf16", kind="gated", step=True, rows=16384, width=4096, act="silu", dtype="bf16", bits=8, block=64),
        # Weight gradients of active linear layers from the 8-bit cache of their input: the feed-forward's first matrix for
        # the largest batch, its second in fp32 for 64 images of 197 tokens, and a head of an odd number of classes.
        dict(name="weight_bf16", kind="weight", rows=16384, outputs=4096, inputs=1024, dtype="bf16", bits=8, block=64),
        dict(name="weight_f32", kind="weight", rows=12608, outputs=1024, inputs=4096, dtype="f32", bits=8, block=64),
        dict(name="weight_odd_bf16", kind="weight", rows=4099, outputs=1003, inputs=768, dtype="bf16", bits=4, block=32),
    ]


MOST_HEADS = 16384 * 48 * 128              # elements of the largest listed case of each kind, and multiplications
MOST_GATED = 16384 * 8192
MOST_WEIGHT = 16384 * 4096 * 1024


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["heads", "gated", "weight"])
    case = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]))
    if kind == "heads":
        dim = rng.choice([32, 64, 80, 96, 128, 192, 256])
        kv = rng.choice([1, 2, 4, 8, 12, 16])
        q = kv * rng.choice([1, 1, 2, 4, 7] if kv <= 4 else [1, 2])
        most = MOST_HEADS // ((q + 2 * kv) * dim * (1 if case["dtype"] == "bf16" else 2))
        step = rng.random() < 0.7
        tokens = 1 if not step and rng.random() < 0.5 else _log_int(rng, 1, min(4096, most))
        blocks = [b for b in (32, 64, 128, 256) if dim % b == 0]
        bits = rng.choice([8, 8, 4, 0]) if step and blocks else 0
        case.update(step=step, batch=_log_int(rng, 1, max(1, min(512 if tokens == 1 else 16384, most // tokens))), tokens=tokens, q_heads=q,
                    kv_heads=kv, dim=dim, rotary=rng.choice([dim, dim, dim // 32 * 16, 0]), adjacent=rng.random() < 0.3,
                    norm=rng.random() < 0.8, ids=rng.choice(["none", "far", "padded"]), bits=bits, block=rng.choice(blocks) if bits else 0)
        if case["rotary"] == 0:
            case["norm"] = True
        if not case["norm"]:
            case.update(bits=0, block=0)
    elif kind == "gated":
        step = rng.random() < 0.8
        bits = rng.choice([8, 8, 4]) if step else 0
        block = rng.choice([32, 64, 128, 256]) if bits else 0
        unit = block or 8
        width = unit * _log_int(rng, max(1, 128 // unit), 8192 // unit)
        most = MOST_GATED // (2 * width * (1 if case["dtype"] == "bf16" else 2))
        case.update(step=step, rows=_log_int(rng, 1, min(16384, most)), width=width, act=rng.choice(["silu", "gelu"]), bits=bits, block=block)
    else:
        block = rng.choice([32, 64, 128, 256])
        inputs = block * _log_int(rng, max(1, 128 // block), 4096 // block)
        outputs = _log_int(rng, 2, 4096)
        rows = _log_int(rng, 1, 16384)
        most = MOST_WEIGHT // (inputs * outputs * (1 if case["dtype"] == "bf16" else 2))
        case.update(rows=min(rows, max(1, most)), outputs=outputs, inputs=inputs, bits=rng.choice([8, 8, 4]), block=block)
    return case


# ------------------------------------------------------------------------------------------------------- inputs

def _activation(g, rows, cols):
    """N(0, 1) with one element in a thousand twenty times as large."""
    x = torch.randn(rows, cols, generator=g, device=DEV)
    hit = torch.randint(0, 1000, (rows, cols), generator=g, device=DEV, dtype=torch.int16) == 0
    return torch.where(hit, x * 20.0, x)


def _cache_buffers(n, bits, block):
    return (torch.empty(n * bits // 8, dtype=torch.uint8, device=DEV) if bits else None,
            torch.empty(n // block, dtype=torch.float32, device=DEV) if bits else None)


def _packed(code, bits):
    """The bytes that whole numbers are kept in: 8 bits, or two to a byte, the first in the low half."""
    code = code.to(torch.int8).view(torch.uint8).view(-1)
    return code if bits == 8 else (code[0::2] & 15) | (code[1::2] << 4)


def _quantised(x, bits, block):
    """(code, scale) of runs of ``block`` elements, in 32 bits as the cache is defined: multiplied by qmax / max|x| and rounded
    to even; a run of zeros, or one whose factor overflows, is kept as zeros."""
    qmax = 2 ** (bits - 1) - 1
    x = x.float().reshape(-1, block)
    top = x.abs().amax(1, keepdim=True)
    whole = torch.full_like(top, qmax)                     # a quotient by a number is multiplied by its reciprocal: two roundings
    factor = whole / top
    kept = torch.isfinite(factor)
    code = (x * torch.where(kept, factor, 0.0)).round().clamp(-qmax - 1, qmax)
    return code, torch.where(kept, top / whole, 0.0)


def _unpacked(codes, bits):
    if bits == 8:
        return codes.view(torch.int8).float()
    both = torch.stack((codes & 15, codes >> 4), -1).view(-1).to(torch.int16)
    return torch.where(both > 7, both - 16, both).float()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    s = dict(case=case)
    if case["kind"] == "heads":
        B, T, Hq, Hk, D, R = (case[k] for k in ("batch", "tokens", "q_heads", "kv_heads", "dim", "rotary"))
        s["qkv"] = _activation(g, B * T, (Hq + 2 * Hk) * D).to(dtype).view(B, T, -1)
        s["gamma_q"] = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEV) if case["norm"] else None
        s["gamma_k"] = 1.0 + 0.1 * torch.randn(D, generator=g, device=DEV) if case["norm"] else None
        s["ids"] = None
        places = T
        if case["ids"] != "none":                          # where each token stands; padding (-1) is not turned
            places = max(T, 8192)
            first = torch.randint(0, places - T + 1, (B, 1), generator=g, device=DEV)
            ids = first + torch.arange(T, device=DEV)
            if case["ids"] == "padded":
                length = torch.randint(T // 2, T + 1, (B, 1), generator=g, device=DEV)
                ids = torch.where(torch.arange(T, device=DEV) < length, ids, -1)
            s["ids"] = ids.to(torch.int32).contiguous()
        s["table"] = None
        if R:                                              # cosines, then sines, of each place's angles
            angle = torch.arange(places, device=DEV, dtype=torch.float64)[:, None] * ROTARY_BASE ** (
                -torch.arange(0, R, 2, device=DEV, dtype=torch.float64) / R)
            s["table"] = torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()
        s["q_scale"] = 1.0 / math.sqrt(D)
        s["q"] = torch.empty(B, Hq, T, D, dtype=dtype, device=DEV)
        s["kt"] = torch.empty(B, Hk, D, T, dtype=dtype, device=DEV)
        s["v"] = torch.empty(B, Hk, T, D, dtype=dtype, device=DEV)
        s["rstd"] = torch.empty(B * T, Hq + Hk, device=DEV) if case["norm"] else None
        s["codes"], s["scales"] = _cache_buffers(B * T * (Hq + Hk) * D, case["bits"], case["block"])
        if case["step"]:
            s["dq"], s["dkt"], s["dv"] = ((torch.randn(t.shape, generator=g, device=DEV) * 0.1).to(dtype) for t in (s["q"], s["kt"], s["v"]))
            s["dqkv"] = torch.empty_like(s["qkv"])
            s["dgamma_q"], s["dgamma_k"] = (torch.empty(D, device=DEV) if case["norm"] else None for _ in range(2))
    elif case["kind"] == "gated":
        rows, F = case["rows"], case["width"]
        s["x"] = _activation(g, rows, 2 * F).to(dtype)
        s["y"] = torch.empty(rows, F, dtype=dtype, device=DEV)
        s["codes"], s["scales"] = _cache_buffers(rows * 2 * F, case["bits"], case["block"])
        if case["step"]:
            s["dy"] = (torch.randn(rows, F, generator=g, device=DEV) * 0.1).to(dtype)
            s["dx"] = torch.empty_like(s["x"])
    else:                                                  # what the forward pass left: the cache, and the gradient that arrives
        M, N, K = case["rows"], case["outputs"], case["inputs"]
        code, scale = _quantised(_activation(g, M, K).to(dtype), case["bits"], case["block"])
        s["codes"], s["scales"] = _packed(code, case["bits"]).contiguous(), scale.view(-1)
        s["dy"] = (torch.randn(M, N, generator=g, device=DEV) * 0.1).to(dtype)
        s["dw"] = torch.empty(N, K, dtype=dtype, device=DEV)
    return s


# -------------------------------------------------------------------------------------------------- plain forms

def _turn(y, cos, sin, adjacent):
    """The first elements of each row in pairs (a, b) -> (a cos - b sin, b cos + a sin); cos, sin (batch, tokens, 1, pairs)."""
    R = 2 * cos.shape[-1]
    if adjacent:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., : R // 2], y[..., R // 2 : R]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, y[..., R:]), -1)


def _angles(s):
    """(cos, sin) of every token, 1 and 0 where its place is not in the table."""
    B, T = s["qkv"].shape[:2]
    half = s["table"].shape[1] // 2
    ids = torch.arange(T, device=DEV).expand(B, T) if s["ids"] is None else s["ids"].long()
    inside = ((ids >= 0) & (ids < s["table"].shape[0]))[..., None]
    row = s["table"][torch.where(inside[..., 0], ids, 0)]
    return torch.where(inside, row[..., :half], 1.0)[:, :, None], torch.where(inside, row[..., half:], 0.0)[:, :, None]


def _plain_heads(s):
    case = s["case"]
    B, T, Hq, Hk, D = (case[k] for k in ("batch", "tokens", "q_heads", "kv_heads", "dim"))
    dtype = s["qkv"].dtype
    x = s["qkv"].float().view(B, T, Hq + 2 * Hk, D)
    qk = x[:, :, : Hq + Hk]
    y = qk
    if case["norm"]:
        rstd = 1.0 / torch.sqrt(qk.square().mean(-1, keepdim=True) + EPS)
        gamma = torch.cat((s["gamma_q"].expand(Hq, D), s["gamma_k"].expand(Hk, D)))
        y = qk * rstd * gamma
    if case["rotary"]:
        cos, sin = _angles(s)
        y = _turn(y, cos, sin, case["adjacent"])
    out = dict(q=(y[:, :, :Hq] * s["q_scale"]).transpose(1, 2).to(dtype).contiguous(), kt=y[:, :, Hq:].permute(0, 2, 3, 1).to(dtype).contiguous(),
               v=s["qkv"].view(B, T, -1, D)[:, :, Hq + Hk :].transpose(1, 2).contiguous())
    if not case["step"]:
        return out
    if case["bits"]:
        code, scale = _quantised(qk, case["bits"], case["block"])
        qk = (code * scale).view(qk.shape)
    grad = torch.cat((s["dq"].float().transpose(1, 2) * s["q_scale"], s["dkt"].float().permute(0, 3, 1, 2)), 2)
    if case["rotary"]:
        grad = _turn(grad, cos, -sin, case["adjacent"])
    if case["norm"]:
        xn = qk * rstd
        by = (grad * xn).view(B * T, Hq + Hk, D)
        out["dgamma_q"], out["dgamma_k"] = by[:, :Hq].sum((0, 1)), by[:, Hq:].sum((0, 1))
        grad = grad * gamma
        grad = rstd * (grad - xn * (grad * xn).mean(-1, keepdim=True))
    out["dqkv"] = torch.cat((grad.to(dtype), s["dv"].transpose(1, 2)), 2).view(B, T, -1)
    return out


def _act_and_slope(g, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    p = 0.5 * torch.erfc(g * -math.sqrt(0.5))
    return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def _plain_gated(s):
    case = s["case"]
    F = case["width"]
    x = s["x"].float()
    out = dict(y=(_act_and_slope(x[:, :F], case["act"])[0] * x[:, F:]).to(s["x"].dtype))
    if case["step"]:
        code, scale = _quantised(x, case["bits"], case["block"])
        x, dy = (code * scale).view(x.shape), s["dy"].float()
        value, slope = _act_and_slope(x[:, :F], case["act"])
        out["dx"] = torch.cat((dy * x[:, F:] * slope, dy * value), 1).to(s["x"].dtype)
    return out


def _plain_weight(s):
    case = s["case"]
    x = (_unpacked(s["codes"], case["bits"]).view(-1, case["block"]) * s["scales"][:, None]).view(case["rows"], case["inputs"])
    return dict(dw=torch.mm(s["dy"].float().t(), x).to(s["dy"].dtype))


# ------------------------------------------------------------------------------------------------------ one pass

def _own_heads(s):
    from paper_2305_18513_amd import binding as sf
    case = s["case"]
    pairs = sf.ROTARY_ADJACENT if case["adjacent"] else sf.ROTARY_HALVES
    sf.heads_norm_rotate_forward(s["qkv"], s["gamma_q"], s["gamma_k"], EPS, s["table"], pairs, s["ids"], s["q_scale"], case["bits"], case["block"],
                                 s["q"], s["kt"], s["v"], s["rstd"], s["codes"], s["scales"])
    out = dict(q=s["q"], kt=s["kt"], v=s["v"])
    if case["step"]:
        sf.heads_norm_rotate_backward(s["dq"], s["dkt"], s["dv"], None if case["bits"] or not case["norm"] else s["qkv"], s["codes"], s["scales"],
                                      case["bits"], case["block"], s["rstd"], s["gamma_q"], s["gamma_k"], s["table"], pairs, s["ids"],
                                      s["q_scale"], s["dqkv"], s["dgamma_q"], s["dgamma_k"])
        out["dqkv"] = s["dqkv"]
        if case["norm"]:
            out["dgamma_q"], out["dgamma_k"] = s["dgamma_q"], s["dgamma_k"]
    return out


def _own_gated(s):
    from paper_2305_18513_amd import binding as sf
    case = s["case"]
    act = sf.ACT_SILU if case["act"] == "silu" else sf.ACT_GELU
    sf.gated_quant_pack(s["x"], act, sf.Q_BLOCK, case["bits"], case["block"], 0, s["y"], s["codes"], s["scales"])
    if not case["step"]:
        return dict(y=s["y"])
    sf.gated_backward_dequant(s["codes"], s["scales"], act, sf.Q_BLOCK, case["bits"], case["block"], 0, s["dy"], s["dx"])
    return dict(y=s["y"], dx=s["dx"])


def _own_weight(s):
    from paper_2305_18513_amd import binding as sf
    sf.weight_grad_dequant(s["dy"], s["codes"], s["scales"], s["case"]["bits"], s["case"]["block"], s["dw"])
    return dict(dw=s["dw"])


def run(s):
    kind = s["case"]["kind"]
    if kind == "heads":
        return _own_heads(s) if own else _plain_heads(s)
    if kind == "gated":
        return _own_gated(s) if own else _plain_gated(s)
    return _own_weight(s) if own else _plain_weight(s)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2

    def cache(n):
        return n * (case["bits"] / 8 + 4 / case["block"]) if case["bits"] else 0

    if case["kind"] == "heads":
        rows, Hq, Hk, D = case["batch"] * case["tokens"], case["q_heads"], case["kv_heads"], case["dim"]
        every, normed = rows * (Hq + 2 * Hk) * D, rows * (Hq + Hk) * D
        table = 4 * case["rotary"] * min(rows, 8192) + (4 * rows if case["ids"] != "none" else 0)
        moved, flops = 2 * every * e + table + cache(normed), 8 * normed
        if case["norm"]:
            moved += 4 * rows * (Hq + Hk)
        if case["step"]:
            moved += 2 * every * e + table + ((cache(normed) or normed * e) + 4 * rows * (Hq + Hk) if case["norm"] else 0)
            flops += 14 * normed
        return dict(bytes=moved, flops=flops)
    if case["kind"] == "gated":
        n = case["rows"] * case["width"]
        return dict(bytes=3 * n * e + (2 * cache(2 * n) + 3 * n * e if case["step"] else 0), flops=(30 if case["step"] else 10) * n)
    M, N, K = case["rows"], case["outputs"], case["inputs"]
    return dict(bytes=M * N * e + cache(M * K) + N * K * e, flops=2 * M * N * K)


# ------------------------------------------------------------------------------------------------ in 64 bits

def _kept(x, bits, block):
    """What a cache of x gives back.  Its codes are whole numbers that 32-bit arithmetic defines (a quotient, a product, a rounding
    each); their values are formed in 64."""
    runs = x.float().reshape(-1, block)
    top = torch.max(runs.abs(), 1, keepdim=True).values
    most = float(2 ** (bits - 1) - 1)
    most_of = torch.full_like(top, most)
    factor = most_of / top
    fine = factor < math.inf
    whole = torch.clamp(torch.round(runs * torch.where(fine, factor, torch.zeros_like(top))), -most - 1.0, most)
    return (whole.double() * torch.where(fine, top / most_of, torch.zeros_like(top)).double()).view(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "weight":
        M, K = case["rows"], case["inputs"]
        if case["bits"] == 8:
            code = s["codes"].to(torch.int16)
        else:
            code = torch.empty(M * K, dtype=torch.int16, device=DEV)
            code[0::2], code[1::2] = s["codes"] % 16, s["codes"] // 16
        code = code - (code >= 2 ** (case["bits"] - 1)).to(torch.int16) * 2 ** case["bits"]
        x = code.double().view(M, K) * s["scales"].double().repeat_interleave(case["block"]).view(M, K)
        return dict(dw=s["dy"].double().t() @ x)
    if case["kind"] == "gated":
        def parts(x):
            gate, up = x.double().chunk(2, 1)
            if case["act"] == "silu":
                p = torch.sigmoid(gate)
                return gate * p, p + gate * p * torch.sigmoid(-gate), up
            p = torch.special.ndtr(gate)
            return gate * p, p + gate * torch.exp(-gate.square() / 2) * (2 * math.pi) ** -0.5, up

        value, _, up = parts(s["x"])
        out = dict(y=value * up)
        if case["step"]:
            value, slope, up = parts(_kept(s["x"], case["bits"], case["block"]))
            out["dx"] = torch.cat((s["dy"].double() * slope * up, s["dy"].double() * value), 1)
        return out
    B, T, Hq, Hk, D, R = (case[k] for k in ("batch", "tokens", "q_heads", "kv_heads", "dim", "rotary"))
    # each token's pairs as complex numbers times e^(i angle)
    unit = None
    if R:
        wave = torch.complex(s["table"][:, : R // 2].double(), s["table"][:, R // 2 :].double())
        wave = torch.cat((wave, torch.ones(1, R // 2, dtype=wave.dtype, device=DEV)))          # the last row turns nothing
        ids = torch.arange(T, device=DEV).repeat(B, 1) if s["ids"] is None else s["ids"].long()
        ids = torch.where((ids < 0) | (ids >= len(wave) - 1), len(wave) - 1, ids)
        unit = wave[ids].view(B, T, 1, R // 2)

    def turn(y, unit):
        if unit is None:
            return y
        first = y[..., :R].unflatten(-1, (R // 2, 2) if case["adjacent"] else (2, R // 2))
        first = first if case["adjacent"] else first.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(first.contiguous()) * unit)
        z = z if case["adjacent"] else z.transpose(-1, -2)
        return torch.cat((z.flatten(-2), y[..., R:]), -1)

    qk, v = s["qkv"].view(B, T, -1, D).split((Hq + Hk, Hk), 2)
    x = qk.double()
    gain, rstd = 1.0, 1.0
    if case["norm"]:
        rstd = (x.square().sum(-1, keepdim=True) / D + EPS) ** -0.5
        gain = torch.stack([s["gamma_q"]] * Hq + [s["gamma_k"]] * Hk).double()
    y = turn(x * rstd * gain, unit)
    out = dict(q=y[:, :, :Hq].permute(0, 2, 1, 3) * s["q_scale"], kt=y[:, :, Hq:].permute(0, 2, 3, 1), v=v.permute(0, 2, 1, 3))
    if case["step"]:
        dq, dk = s["dq"].double().permute(0, 2, 1, 3) * s["q_scale"], s["dkt"].double().permute(0, 3, 1, 2)
        d = turn(torch.cat((dq, dk), 2), None if unit is None else unit.conj())
        if case["norm"]:
            xn = (_kept(qk.contiguous(), case["bits"], case["block"]) if case["bits"] else x) * rstd
            out["dgamma_q"], out["dgamma_k"] = ((d * xn)[:, :, h].sum((0, 1, 2)) for h in (slice(0, Hq), slice(Hq, None)))
            d = d * gain
            d = (d - xn * ((d * xn).sum(-1, keepdim=True) / D)) * rstd
        out["dqkv"] = torch.cat((d, s["dv"].double().permute(0, 2, 1, 3)), 2).reshape(B, T, -1)
    return out
