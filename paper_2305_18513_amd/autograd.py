"""torch.autograd wrappers over the C ABI (Alg. 4 and Sec. 4 of the paper).

Each Function runs its forward through the library, keeps only the compressed
form of the activation its backward needs, and skips the weight gradient of a
frozen layer.  Nothing here computes on its own what a kernel of the library
computes; the dense matrix products of the linear layers are the library's for
fp32 operands of sizes at which it is the quicker one, and torch's otherwise.

  GeluFunction       y = GELU(x); caches x in `bits` bits (per-block scales);
                     backward multiplies by GELU'(x^) straight from the cache.
  LayerNormFunction  frozen: caches the `keep_ppm` largest |x~| of the whole
                     tensor with int32 indices, row pointers and rstd; backward
                     is the paper's input-gradient formula on those pairs, and
                     gamma / beta get no gradient.  Active: caches x exactly
                     and returns all three gradients.  With `quant_bits` the
                     cache is instead the block-scaled codes of x written by the
                     forward kernel itself (plus mean and rstd); backward rebuilds
                     x^ in registers, and an active layer's gamma / beta gradients
                     use the dequantised x^.
  SoftmaxFunction    p = softmax(logits) over the last dimension (at most 2048
                     wide); caches the `keep_ppm` largest probabilities of every
                     row with uint16 columns; backward is the derivative of
                     softmax with the restored (sparse) row in place of p.
  SoftmaxMatmulFunction  out = softmax(logits) @ V with the probabilities shared
                     between the two ops as the paper has it: only the kept
                     pairs and V are cached.  Backward: dP = dO @ V^T (dense
                     product, torch's), dV = P^^T @ dO with P^ restored from the
                     pairs, dlogits from the pairs as in SoftmaxFunction.
  GatedFunction      y = act(gate) * up of rows [gate | up]; caches them in `bits`
                     bits, or nothing where no gradient is asked for; backward from
                     the cache.
  HeadsNormRotateFunction  (q, k^T, v) as SplitHeadsFunction, keys and values shared by
                     groups of query heads, each query and key head normed and
                     turned by its token's position in the same pass; caches the
                     query and key columns in `bits` bits (0: keeps the rows
                     themselves) and rstd; norms that are frozen get no gradients.
  AttentionFunction  softmax(scale q k^T + bias) v over rows of any length, the probabilities formed
                     again in the backward pass: it keeps its operands, its output and
                     two numbers a query.  The bias is a learned table by buckets of the
                     distance, or none; a frozen table gets no gradient.
  SelfAttentionFunction  the same from the rows of a QKV projection, as they lie.
  SplitHeadsFunction (q, k^T, v) of the attention products from the rows of a QKV
                     projection in one pass, their gradients back in another.
  MatmulFunction     out = a @ b with both operands cached in 8 bits (the paper's
                     placement for MatMul's activations).
  LinearFunction     the freezing rule of Alg. 4: a layer whose weight does not
                     require a gradient (frozen by the scheduler) keeps nothing of
                     its input and returns no weight gradient; an active one keeps
                     its input in `bits` bits and forms the weight gradient from
                     the dequantised input (`straight`: from the codes themselves,
                     by the library's own product, where a block lies in one row).

A backward pass may be captured into a HIP graph once no eager graph of the same leaves is alive (with one, the process
has ended in torch's end of the capture, probably because the engine ties the capture to the eager one's stream): capture
the first pass on a side stream after a warm-up there, as torch's own notes have it, and let go of every loss computed before.

All tensors are CUDA tensors (fp32 or bf16 activations; gamma / beta and the
kept standardised values fp32); the kernels run on torch's current stream.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding as sf


def _flat(t: torch.Tensor) -> torch.Tensor:
    return t.contiguous().view(-1)


def _quantise(t: torch.Tensor, bits: int, block: int):
    """(codes, scales) of the flattened tensor, block-scaled."""
    f = _flat(t)
    n = f.numel()
    codes = torch.empty(sf.packed_bytes(n, bits), dtype=torch.uint8, device=t.device)
    scales = torch.empty(sf.num_blocks(n, block), dtype=torch.float32, device=t.device)
    sf.quant_pack(f, sf.Q_BLOCK, bits, block, 0, codes, scales)
    return codes, scales


def _dequantise(codes, scales, bits: int, block: int, shape, dtype) -> torch.Tensor:
    out = torch.empty(shape, dtype=dtype, device=codes.device)
    sf.dequant_unpack(codes, scales, sf.Q_BLOCK, bits, block, 0, out.view(-1))
    return out


def _right(t: torch.Tensor) -> torch.Tensor:
    """The right operand of a batched product, laid out for bf16: torch's bf16 product has faulted the GPU where it was a
    transposed view."""
    return t.contiguous() if t.dtype == torch.bfloat16 else t


class MatmulFunction(torch.autograd.Function):
    """out = a @ b with both operands cached in `bits` bits (the paper keeps MatMul's activations in 8 bits);
    backward multiplies the incoming gradient with the dequantised operands."""

    @staticmethod
    def forward(ctx, a: torch.Tensor, b: torch.Tensor, bits: int = 8, block: int = 64):
        out = torch.matmul(a, _right(b))
        ca, sa = _quantise(a, bits, block)
        cb, sb = _quantise(b, bits, block)
        ctx.save_for_backward(ca, sa, cb, sb)
        ctx.meta = (bits, block, a.shape, b.shape, a.dtype)
        return out

    @staticmethod
    def backward(ctx, grad_output: torch.Tensor):
        ca, sa, cb, sb = ctx.saved_tensors
        bits, block, sha, shb, dtype = ctx.meta
        b_hat = _dequantise(cb, sb, bits, block, shb, dtype)
        da = torch.matmul(grad_output, _right(b_hat.transpose(-1, -2)))
        del b_hat
        a_hat = _dequantise(ca, sa, bits, block, sha, dtype)
        db = torch.matmul(a_hat.transpose(-1, -2), _right(grad_output))
        return da, db, None, None


class GeluFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x: torch.Tensor, bits: int = 4, block: int = 64):
        xf = _flat(x)
        n = xf.numel()
        y = torch.empty_like(xf)
        codes = torch.empty(sf.packed_bytes(n, bits), dtype=torch.uint8, device=x.device)
        scales = torch.empty(sf.num_blocks(n, block), dtype=torch.float32, device=x.device)
        sf.gelu_quant_pack(xf, sf.Q_BLOCK, bits, block, 0, y, codes, scales)
        ctx.save_for_backward(codes, scales)
        ctx.quant = (bits, block)
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, grad_output: torch.Tensor):
        codes, scales = ctx.saved_tensors
        bits, block = ctx.quant
        dy = _flat(grad_output)
        dx = torch.empty_like(dy)
        sf.gelu_backward_dequant(codes, scales, sf.Q_BLOCK, bits, block, 0, dy, dx)
        return dx.view(grad_output.shape), None, None


class LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, eps: float = 1e-5,
                frozen: bool = False, keep_ppm: int = 100000, quant_bits: int = 0, block: int = 64):
        H = x.shape[-1]
        x2 = x.contiguous().view(-1, H)
        rows = x2.shape[0]
        y = torch.empty_like(x2)
        mean = torch.empty(rows, dtype=torch.float32, device=x.device)
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
        ctx.frozen = frozen
        ctx.quant = (quant_bits, block)
        if quant_bits:
            n = x2.numel()
            codes = torch.empty(sf.packed_bytes(n, quant_bits), dtype=torch.uint8, device=x.device)
            scales = torch.empty(sf.num_blocks(n, block), dtype=torch.float32, device=x.device)
            sf.layernorm_forward_quant_pack(x2, gamma, beta, eps, quant_bits, block, y, mean, rstd, codes, scales)
            ctx.save_for_backward(codes, scales, mean, rstd, gamma)
            return y.view(x.shape)
        sf.layernorm_forward(x2, gamma, beta, eps, y, mean, rstd)
        if frozen:
            n = x2.numel()
            k = sf.keep_count(n, keep_ppm)
            vals = torch.empty(k, dtype=torch.float32, device=x.device)
            idx = torch.empty(k, dtype=torch.int32, device=x.device)
            row_ptr = torch.empty(rows + 1, dtype=torch.int32, device=x.device)
            if k > 0:
                sf.prune_global_standardized(x2, mean, rstd, k, vals, idx, True, None, row_ptr)
            else:
                row_ptr.zero_()
            ctx.k = k
            ctx.save_for_backward(vals, idx, row_ptr, rstd, gamma)
        else:
            ctx.save_for_backward(x2, mean, rstd, gamma)
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, grad_output: torch.Tensor):
        H = grad_output.shape[-1]
        dy = grad_output.contiguous().view(-1, H)
        none = (None,) * 5
        bits, block = ctx.quant
        if bits:
            codes, scales, mean, rstd, gamma = ctx.saved_tensors
            dx = torch.empty_like(dy)
            sf.layernorm_backward_dequant(codes, scales, bits, block, mean, rstd, gamma, dy, dx)
            if ctx.frozen:
                return (dx.view(grad_output.shape), None, None) + none
            x_hat = torch.empty_like(dy)
            sf.dequant_unpack(codes, scales, sf.Q_BLOCK, bits, block, 0, x_hat.view(-1))
            dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(gamma)
            sf.layernorm_param_grads(x_hat, mean, rstd, dy, dgamma, dbeta)
            return (dx.view(grad_output.shape), dgamma, dbeta) + none
        if ctx.frozen:
            vals, idx, row_ptr, rstd, gamma = ctx.saved_tensors
            dx = torch.empty_like(dy)
            sf.layernorm_backward_pruned(vals, idx, row_ptr, ctx.k, rstd, gamma, dy, dx)
            return (dx.view(grad_output.shape), None, None) + none
        x2, mean, rstd, gamma = ctx.saved_tensors
        dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(gamma)
        sf.layernorm_param_grads(x2, mean, rstd, dy, dgamma, dbeta)
        dx = torch.empty_like(dy)
        sf.layernorm_backward(x2, mean, rstd, gamma, dy, dx)
        return (dx.view(grad_output.shape), dgamma, dbeta) + none


class SoftmaxFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits: torch.Tensor, keep_ppm: int = 100000):
        cols = logits.shape[-1]
        l2 = logits.contiguous().view(-1, cols)
        rows = l2.shape[0]
        k = max(1, sf.keep_count(cols, keep_ppm))
        probs = torch.empty_like(l2)
        vals = torch.empty(rows, k, dtype=l2.dtype, device=l2.device)
        idx = torch.empty(rows, k, dtype=torch.uint16, device=l2.device)
        sf.softmax_prune(l2, k, probs, vals, idx)
        ctx.save_for_backward(vals, idx)
        return probs.view(logits.shape)

    @staticmethod
    def backward(ctx, grad_output: torch.Tensor):
        vals, idx = ctx.saved_tensors
        cols = grad_output.shape[-1]
        dp = grad_output.contiguous().view(-1, cols)
        ds = torch.empty_like(dp)
        sf.softmax_backward_pruned(vals, idx, None, dp, ds)
        return ds.view(grad_output.shape), None


class SoftmaxMatmulFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits: torch.Tensor, v: torch.Tensor, keep_ppm: int = 100000, v_bits: int = 0, block: int = 64):
        # logits (..., Tq, Tk), v (..., Tk, D); v_bits != 0 caches V quantised as well
        cols = logits.shape[-1]
        l2 = logits.contiguous().view(-1, cols)
        rows = l2.shape[0]
        k = max(1, sf.keep_count(cols, keep_ppm))
        probs = torch.empty_like(l2)
        vals = torch.empty(rows, k, dtype=l2.dtype, device=l2.device)
        idx = torch.empty(rows, k, dtype=torch.uint16, device=l2.device)
        sf.softmax_prune(l2, k, probs, vals, idx)
        out = torch.matmul(probs.view(logits.shape), _right(v))
        if v_bits:
            cv, sv = _quantise(v, v_bits, block)
            ctx.save_for_backward(vals, idx, cv, sv)
        else:
            ctx.save_for_backward(vals, idx, v)
        ctx.meta = (logits.shape, v.shape, v.dtype, v_bits, block)
        return out

    @staticmethod
    def backward(ctx, grad_output: torch.Tensor):
        shape, v_shape, v_dtype, v_bits, block = ctx.meta
        if v_bits:
            vals, idx, cv, sv = ctx.saved_tensors
            v = _dequantise(cv, sv, v_bits, block, v_shape, v_dtype)
        else:
            vals, idx, v = ctx.saved_tensors
        cols = shape[-1]
        rows = vals.shape[0]
        if grad_output.dim() > 3:                           # (three dimensions are multiplied as they lie)
            grad_output = grad_output.contiguous()          # both products would lay out a transposed one for themselves
        dp = torch.matmul(grad_output, _right(v.transpose(-1, -2))).contiguous().view(rows, cols)
        p_hat = torch.empty(rows, cols, dtype=vals.dtype, device=vals.device)
        sf.restore_scores(vals, idx, None, p_hat)
        dv = torch.matmul(p_hat.view(shape).transpose(-1, -2), _right(grad_output))
        ds = torch.empty_like(dp)
        sf.softmax_backward_pruned(vals, idx, None, dp, ds)
        return ds.view(shape), dv, None, None, None


class SplitHeadsFunction(torch.autograd.Function):
    """(q, k^T, v) of the attention products from the rows (B, T, 3 * H) of a QKV projection, q times ``q_scale``; backward
    lays the three gradients into one row buffer.  Nothing is kept."""

    @staticmethod
    def forward(ctx, qkv: torch.Tensor, heads: int, q_scale: float):
        B, T, H3 = qkv.shape
        D = H3 // (3 * heads)
        q = torch.empty(B, heads, T, D, dtype=qkv.dtype, device=qkv.device)
        kt = torch.empty(B, heads, D, T, dtype=qkv.dtype, device=qkv.device)
        v = torch.empty_like(q)
        sf.split_heads(qkv.contiguous(), q_scale, q, kt, v)
        ctx.meta = (qkv.shape, q_scale)
        return q, kt, v

    @staticmethod
    def backward(ctx, dq: torch.Tensor, dkt: torch.Tensor, dv: torch.Tensor):
        shape, q_scale = ctx.meta
        dqkv = torch.empty(shape, dtype=dq.dtype, device=dq.device)
        sf.merge_heads(dq.contiguous(), dkt.contiguous(), dv.contiguous(), q_scale, dqkv)
        return dqkv, None, None


def _recorded(ctx) -> bool:
    """Whether the call becomes part of a graph.  Inside forward gradients are off whatever the caller has, and requires_grad and
    needs_input_grad do not tell, but a call under no_grad is linked to nothing.  (A traced context has no links to look at.)"""
    return torch.compiler.is_compiling() or len(ctx.next_functions) > 0


class GatedFunction(torch.autograd.Function):
    """y = act(gate) * up for x = [gate | up] (..., 2 F); ``act`` is binding.ACT_SILU or ACT_GELU, F a multiple of ``block``."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, act: int, bits: int = 8, block: int = 64):
        F = x.shape[-1] // 2
        x2 = x.contiguous().view(-1, x.shape[-1])
        y = torch.empty(x2.shape[0], F, dtype=x.dtype, device=x.device)
        if not (ctx.needs_input_grad[0] and _recorded(ctx)):
            sf.gated_quant_pack(x2, act, sf.Q_BLOCK, 0, block, 0, y, None, None)
            return y.view(*x.shape[:-1], F)
        codes = torch.empty(sf.packed_bytes(x2.numel(), bits), dtype=torch.uint8, device=x.device)
        scales = torch.empty(sf.num_blocks(x2.numel(), block), dtype=torch.float32, device=x.device)
        sf.gated_quant_pack(x2, act, sf.Q_BLOCK, bits, block, 0, y, codes, scales)
        ctx.save_for_backward(codes, scales)
        ctx.meta = (act, bits, block, x.shape)
        return y.view(*x.shape[:-1], F)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_output: torch.Tensor):
        codes, scales = ctx.saved_tensors
        act, bits, block, shape = ctx.meta
        dy = grad_output.contiguous().view(-1, shape[-1] // 2)
        dx = torch.empty(dy.shape[0], shape[-1], dtype=dy.dtype, device=dy.device)
        sf.gated_backward_dequant(codes, scales, act, sf.Q_BLOCK, bits, block, 0, dy, dx)
        return dx.view(shape), None, None, None


class HeadsNormRotateFunction(torch.autograd.Function):
    """(q, k^T, v) of the attention products from the rows (B, T, (heads + 2 * kv_heads) * D) of a QKV projection.  gamma_q, gamma_k
    (both None: no norm), table (None: no rotation; binding.rotary_table), pairing, position_ids: binding.heads_norm_rotate_forward.
    A head's D has to be a multiple of ``block`` where ``bits`` is not 0; without a norm nothing is kept."""

    @staticmethod
    def forward(ctx, qkv: torch.Tensor, gamma_q, gamma_k, heads: int, kv_heads: int, table, pairing: int = sf.ROTARY_HALVES, position_ids=None,
                q_scale: float = 1.0, eps: float = 1e-6, bits: int = 8, block: int = 64):
        B, T, width = qkv.shape
        D = width // (heads + 2 * kv_heads)
        norm = gamma_q is not None
        qkv = qkv.contiguous()
        q = torch.empty(B, heads, T, D, dtype=qkv.dtype, device=qkv.device)
        kt = torch.empty(B, kv_heads, D, T, dtype=qkv.dtype, device=qkv.device)
        v = torch.empty(B, kv_heads, T, D, dtype=qkv.dtype, device=qkv.device)
        keeps = norm and any(ctx.needs_input_grad[:3]) and _recorded(ctx)
        bits = bits if keeps else 0
        rstd = codes = scales = None
        if norm:
            rstd = torch.empty(B * T, heads + kv_heads, dtype=torch.float32, device=qkv.device)
        if bits:
            n = B * T * (heads + kv_heads) * D
            codes = torch.empty(sf.packed_bytes(n, bits), dtype=torch.uint8, device=qkv.device)
            scales = torch.empty(sf.num_blocks(n, block), dtype=torch.float32, device=qkv.device)
        sf.heads_norm_rotate_forward(qkv, gamma_q, gamma_k, eps, table, pairing, position_ids, q_scale, bits, block, q, kt, v, rstd, codes, scales)
        ctx.save_for_backward(qkv if keeps and not bits else None, codes, scales, rstd if keeps else None, gamma_q, gamma_k, table, position_ids)
        ctx.meta = (qkv.shape, pairing, q_scale, bits, block)
        return q, kt, v

    @staticmethod
    @once_differentiable
    def backward(ctx, dq: torch.Tensor, dkt: torch.Tensor, dv: torch.Tensor):
        qkv, codes, scales, rstd, gamma_q, gamma_k, table, position_ids = ctx.saved_tensors
        shape, pairing, q_scale, bits, block = ctx.meta
        dqkv = torch.empty(shape, dtype=dq.dtype, device=dq.device)
        dgamma_q = dgamma_k = None
        if gamma_q is not None and any(ctx.needs_input_grad[1:3]):
            dgamma_q, dgamma_k = (torch.empty_like(g) for g in (gamma_q, gamma_k))
        sf.heads_norm_rotate_backward(dq.contiguous(), dkt.contiguous(), dv.contiguous(), qkv, codes, scales, bits, block, rstd, gamma_q, gamma_k,
                                      table, pairing, position_ids, q_scale, dqkv, dgamma_q, dgamma_k)
        return (dqkv, dgamma_q, dgamma_k) + (None,) * 9


def _attend(ctx, q, k, v, layout, scale, causal, lengths, table, bucket_of, saved):
    """One forward pass; keeps what the backward pass reads (``saved``: what q, k and v are parts of) where it is asked for."""
    apart = layout == sf.HEADS_APART
    B, Tq, Hq, D = (q.shape[i] for i in ((0, 2, 1, 3) if apart else (0, 1, 2, 3)))
    out = torch.empty(B, Tq, Hq, D, dtype=q.dtype, device=q.device)
    stats = torch.empty(B, Hq, Tq, 2, dtype=torch.float32, device=q.device)
    table = None if table is None else table.contiguous()
    sf.attention_forward(q, k, v, layout, scale, causal, lengths, table, bucket_of, out, stats)
    if any(ctx.needs_input_grad) and _recorded(ctx):
        ctx.save_for_backward(*saved, out, stats, lengths, table, bucket_of)
    return out


class AttentionFunction(torch.autograd.Function):
    """out (B, q_tokens, heads, D) of q, k, v.  layout binding.HEADS_ROWS: (B, tokens, heads, D) each; HEADS_APART: (q, k^T, v) as
    SplitHeadsFunction and HeadsNormRotateFunction give them.  causal: query i sees keys j <= i + k_tokens - q_tokens.  lengths
    (int32, B): keys of each sequence; they move neither the causal order nor the distances of the bias, which are counted from k_tokens.
    table (buckets, heads) and bucket_of: binding.attention_forward, binding.distance_buckets."""

    @staticmethod
    def forward(ctx, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: float, causal: bool = False, lengths=None, table=None, bucket_of=None,
                layout: int = sf.HEADS_ROWS):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        ctx.meta = (scale, causal, layout)
        return _attend(ctx, q, k, v, layout, scale, causal, lengths, table, bucket_of, (q, k, v))

    @staticmethod
    @once_differentiable
    def backward(ctx, dout: torch.Tensor):
        q, k, v, out, stats, lengths, table, bucket_of = ctx.saved_tensors
        scale, causal, layout = ctx.meta
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        dtable = torch.empty_like(table) if table is not None and ctx.needs_input_grad[6] else None
        sf.attention_backward(dout.contiguous(), q, k, v, layout, scale, causal, lengths, table, bucket_of, out, stats, dq, dk, dv, dtable)
        return dq, dk, dv, None, None, None, dtable, None, None


class SelfAttentionFunction(torch.autograd.Function):
    """AttentionFunction on the rows (B, T, (heads + 2 * kv_heads) * D) of a QKV projection: queries, keys and values are its columns, the
    gradients come as rows of the same kind, and out is the rows (B, T, heads * D) that the next projection takes."""

    @staticmethod
    def forward(ctx, qkv: torch.Tensor, heads: int, kv_heads: int, scale: float, causal: bool = False, lengths=None, table=None, bucket_of=None):
        B, T, width = qkv.shape
        qkv = qkv.contiguous()
        rows = qkv.view(B, T, heads + 2 * kv_heads, width // (heads + 2 * kv_heads))
        ctx.meta = (heads, kv_heads, scale, causal)
        out = _attend(ctx, *rows.split((heads, kv_heads, kv_heads), 2), sf.HEADS_ROWS, scale, causal, lengths, table, bucket_of, (qkv,))
        return out.view(B, T, out.shape[2] * out.shape[3])

    @staticmethod
    @once_differentiable
    def backward(ctx, dout: torch.Tensor):
        qkv, out, stats, lengths, table, bucket_of = ctx.saved_tensors
        heads, kv_heads, scale, causal = ctx.meta
        B, T, width = qkv.shape
        dqkv = torch.empty_like(qkv)
        parts = [t.view(B, T, heads + 2 * kv_heads, out.shape[3]).split((heads, kv_heads, kv_heads), 2) for t in (qkv, dqkv)]
        dtable = torch.empty_like(table) if table is not None and ctx.needs_input_grad[6] else None
        sf.attention_backward(dout.contiguous().view(out.shape), *parts[0], sf.HEADS_ROWS, scale, causal, lengths, table, bucket_of, out, stats, *parts[1],
                              dtable)
        return dqkv, None, None, None, None, None, dtable, None


def _plain(t: torch.Tensor) -> bool:
    """Whether a kernel may be handed the tensor's memory as it is."""
    return (type(t) in (torch.Tensor, torch.nn.Parameter) and torch._C._has_storage(t) and t.is_cuda
            and t.is_contiguous() and not t.is_neg() and not t._is_zerotensor() and t.data_ptr() % 16 == 0)


def _watched() -> bool:
    """Whether more than the value is asked for, or less: a product to be differentiated (either way), cast, traced or
    intercepted, or one for which the program allows torch fewer than 32 bits."""
    return (torch.is_grad_enabled() or torch.is_autocast_enabled() or torch.compiler.is_compiling() or torch.jit.is_tracing()
            or forward_ad._current_level >= 0 or torch._C._len_torch_dispatch_stack() > 0 or torch._C._len_torch_function_stack() > 0
            # torch.backends.cuda.matmul.fp32_precision, which takes 2.1 us to read, this 0.6
            or torch._C._get_fp32_precision_getter("cuda", "matmul") not in ("none", "ieee"))


_MOST_TILES = (1 << 31) // 512                             # of 128 x 64 that a launch of the library's product can have


def _quicker(M: int, N: int, K: int, transposed: bool) -> bool:
    """Whether the library's product takes the shorter time on the GPU (rows x columns x depth, torch's and this in us).

    It does from about 170 tiles of 128 x 64 on, two for three compute units (1792 x 768 x 768 25.2 and 22.0, 3600 x 384 x 384 19.5 and
    13.4, 4096 x 768 x 3072 140 and 102); fewer torch splits along their depth (2048 x 512 x 2048 35 and 50, 1024 x 768 x 768 14 and
    22, 257 x 256 x 256 5.5 and 9.5).  Weights that lie K x N and are deep need 208 (1500 x 960 x 3072 78 and 81, 3300 x 512 x 2048
    57.1 and 56.0), and a quarter of the tiles at most may be padding (260 x 6144 x 1024 32 and 35, 400 x 6000 x 1024 55 and 42).
    Nor do tall ones of few columns and some depth, which go in tiles of 96 columns (40000 x 64 x 1024 54 and 69, 34000 x 128 x 1536 118 and
    139; 22000 x 128 x 1024, whose tiles have 64, 70 and 45), or one step of depth (17000 x 128 x 32 6.7 and 8.7).
    And where torch does not split: up to 256 x 256 and a depth below 1024, but for the very smallest (256 x 256 x 256 63 and 9.5,
    128 x 128 x 768 88 and 21, 64 x 192 x 64 7.1 and 5.9, 64 x 128 x 64 5.5 and 5.9; of depth 1024 8 and 26)."""
    outputs, tiles = M * N, -(-M // 128) * -(-N // 64)
    if M <= 256 and N <= 256 and 64 <= K < 1024:
        return outputs >= 64 * 192
    if K < 64 or (M > 256 * 128 and N <= 128 and K >= 512):
        return False
    return outputs >= (168 if transposed or K <= 1536 else 208) * 128 * 64 and 4 * outputs >= 3 * 128 * 64 * tiles and tiles <= _MOST_TILES


def _dense(x: torch.Tensor, weight: torch.Tensor, transposed: bool):
    """x @ weight.T or x @ weight over x's last dimension by the library's fp32 product, or None where that is torch's."""
    if x.dtype != torch.float32 or weight.dtype != torch.float32 or x.dim() < 2 or weight.dim() != 2:
        return None
    K = x.shape[-1]
    N, depth = weight.shape if transposed else weight.shape[::-1]
    if depth != K or K == 0 or K % 32 != 0:
        return None
    M = x.numel() // K
    if not _quicker(M, N, K, transposed) or _watched() or not (_plain(x) and _plain(weight)):
        return None
    if not (x.get_device() == weight.get_device() == torch.cuda.current_device()):
        return None                                        # the library launches on the current device
    y = torch.empty(*x.shape[:-1], N, dtype=x.dtype, device=x.device)
    sf.product(x.view(M, K), weight, transposed, y.view(M, N))
    return y


class LinearFunction(torch.autograd.Function):
    """y = x W^T (+ b) under the freezing rule of Alg. 4.  Whether the layer is frozen is read off the weight itself
    (``weight.requires_grad``, which is what an inter-layer scheduler flips between iterations): a frozen layer
    keeps nothing of x and produces no weight gradient; an active one keeps x as ``bits``-bit block-scaled codes
    and forms its weight gradient from the dequantised x^.  The library's fp32 product (sizes: ``_quicker``) holds all bits of
    its operands and is no further from the exact one than fp32 additions in any order; where the program allows torch fewer
    bits (``torch.set_float32_matmul_precision``) the products are torch's.  ``straight``: the weight gradient is formed from
    the codes themselves where the layer's inputs are a multiple of ``block``; x^ is not written to memory (sums that are shared
    out take a workspace in its place, of its size or of 256 MiB at most)."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, weight: torch.Tensor, bias, bits: int = 8, block: int = 64, straight: bool = False):
        y = _dense(x, weight, True) if bias is None else None
        if y is None:
            y = torch.nn.functional.linear(x, weight, bias)
        ctx.cache = None                                   # descriptor of what is kept of x: nothing, or (bits, block, shape, dtype)
        ctx.bias_active = bias is not None and bias.requires_grad
        if weight.requires_grad and _recorded(ctx):
            codes, scales = _quantise(x, bits, block)
            ctx.cache = (bits, block, x.shape, x.dtype)
            ctx.straight = straight
            ctx.save_for_backward(weight, codes, scales)
        else:
            ctx.save_for_backward(weight)
        return y

    @staticmethod
    def backward(ctx, dy: torch.Tensor):
        weight = ctx.saved_tensors[0]
        dx = None
        if ctx.needs_input_grad[0]:
            dx = _dense(dy, weight, False)
            if dx is None:
                dx = dy.matmul(weight)
        dy2 = dy.reshape(-1, dy.shape[-1])
        dw = None
        if ctx.cache is not None:
            bits, block, shape, dtype = ctx.cache
            codes, scales = ctx.saved_tensors[1:]
            if ctx.straight:
                dw = _straight(dy2, codes, scales, bits, block, shape[-1], dtype)
            if dw is None:
                dw = dy2.t().mm(_dequantise(codes, scales, bits, block, shape, dtype).view(-1, shape[-1]))
        db = dy2.sum(0) if ctx.bias_active else None
        return dx, dw, db, None, None, None


def _straight(dy: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, bits: int, block: int, K: int, dtype):
    """dy.T @ x^ from x's codes, or None where that is torch's: blocks that straddle rows, types that differ, products that are
    watched, tensors that are not the kernel's to read, gradients past what a call takes."""
    N = dy.shape[1]
    if max(N, K) > 1 << 20 or -(-N // 128) * -(-K // 32) > 1 << 23:
        return None
    if K % block != 0 or dy.dtype != dtype or _watched() or dy.get_device() != torch.cuda.current_device():
        return None
    dy = dy.contiguous()
    if not all(_plain(t) for t in (dy, codes, scales)):
        return None
    dw = torch.empty(N, K, dtype=dtype, device=dy.device)
    sf.weight_grad_dequant(dy, codes, scales, bits, block, dw)
    return dw


def _rows_of_vectors(dim: int, t: torch.Tensor) -> bool:
    """Whether a head's elements are whole 16-byte vectors, which is what split_heads and merge_heads move."""
    return dim * t.element_size() % 16 == 0


def _halves(dim: int) -> bool:
    """Whether sqrt(dim) is a power of two."""
    return dim > 0 and dim & (dim - 1) == 0 and dim.bit_length() % 2 == 1


def encoder_block_params(hidden: int, device="cuda", seed: int = 0, dtype=torch.float32):
    """Random weights of one encoder block (QKV, projection, two feed-forward matrices, two LayerNorms)."""
    g = torch.Generator(device=device).manual_seed(seed)

    def mat(rows, cols):
        return torch.nn.Parameter((torch.randn(rows, cols, generator=g, device=device) * 0.03).to(dtype))

    def vec(value):
        return torch.nn.Parameter(torch.full((hidden,), value, device=device))

    return {"wqkv": mat(3 * hidden, hidden), "wo": mat(hidden, hidden), "w1": mat(4 * hidden, hidden),
            "w2": mat(hidden, 4 * hidden), "g1": vec(1.0), "b1": vec(0.0), "g2": vec(1.0), "b2": vec(0.0)}


def _only_recomputed(*given) -> None:
    """A block that keeps its probabilities has no lengths and no position bias: given ones are refused, not passed over."""
    if any(x is not None for x in given):
        raise ValueError("lengths, bias_table and bucket_of go with recompute")


def frozen_encoder_block(x: torch.Tensor, p: dict, heads: int, wrapped: bool, keep_ppm: int = 100000,
                         gelu_bits: int = 4, block: int = 64, recompute: bool = False, lengths=None, bias_table=None, bucket_of=None) -> torch.Tensor:
    """One pre-LN encoder block whose layers are all frozen: with ``wrapped`` the activations kept
    for the backward pass are the compressed ones (pruned LayerNorm input, pruned attention probabilities shared by
    Softmax and MatMul, 4-bit GELU input, nothing for the frozen linear layers); without, plain torch ops.  With ``wrapped``,
    ``recompute`` keeps no probabilities: attention forms them again, from the projection's rows, and takes the sequences'
    ``lengths`` and a position bias (SelfAttentionFunction)."""
    if not (wrapped and recompute):
        _only_recomputed(lengths, bias_table, bucket_of)
    B, T, H = x.shape
    D = H // heads
    F = torch.nn.functional

    def split(t):
        return t.reshape(B, T, heads, D).transpose(1, 2)

    if wrapped:
        w = {name: t.detach() for name, t in p.items()}    # frozen: the scheduler has switched their gradients off
        h = LayerNormFunction.apply(x, p["g1"], p["b1"], 1e-5, True, keep_ppm)
        qkv = LinearFunction.apply(h, w["wqkv"], None, 8, block)
        if recompute:
            a = SelfAttentionFunction.apply(qkv, heads, heads, 1.0 / D ** 0.5, False, lengths, bias_table, bucket_of)
        elif _rows_of_vectors(D, qkv):
            # 1 / sqrt(D) goes onto q where it is a power of two: that commutes with every rounding on the way (entries of q
            # or its gradient below 1e-35 apart, which may become subnormal or leave the 8-bit cache's range), so these are
            # the numbers of the divided products.  Any other divides them.  (32 x 128 x 768, fp32, forward and backward: heads
            # of 32 1442 -> 1383 us, 64 1360 -> 1290, 96 1325 -> 1276, 128 1328 -> 1260.)
            on_q = _halves(D)
            q, kt, v = SplitHeadsFunction.apply(qkv, heads, 1.0 / D ** 0.5 if on_q else 1.0)
            s = MatmulFunction.apply(q, kt, 8, block)
            s = s if on_q else s / D ** 0.5
        else:
            q, k_, v = qkv.chunk(3, dim=-1)
            s = MatmulFunction.apply(split(q).contiguous(), split(k_).transpose(-1, -2).contiguous(), 8, block) / D ** 0.5
            v = split(v).contiguous()
        if not recompute:
            a = SoftmaxMatmulFunction.apply(s, v, keep_ppm, 8, block).transpose(1, 2).reshape(B, T, H)
        y = x + LinearFunction.apply(a, w["wo"], None, 8, block)
        h = LayerNormFunction.apply(y, p["g2"], p["b2"], 1e-5, True, keep_ppm)
        h = LinearFunction.apply(h, w["w1"], None, 8, block)
        h = LinearFunction.apply(GeluFunction.apply(h, gelu_bits, block), w["w2"], None, 8, block)
        return y + h
    h = F.layer_norm(x, (H,), p["g1"].to(x.dtype), p["b1"].to(x.dtype), 1e-5)
    q, k_, v = F.linear(h, p["wqkv"]).chunk(3, dim=-1)
    s = torch.matmul(split(q), split(k_).transpose(-1, -2)) / D ** 0.5
    a = torch.matmul(torch.softmax(s, -1), split(v)).transpose(1, 2).reshape(B, T, H)
    y = x + F.linear(a, p["wo"])
    h = F.layer_norm(y, (H,), p["g2"].to(x.dtype), p["b2"].to(x.dtype), 1e-5)
    h = F.linear(F.gelu(F.linear(h, p["w1"])), p["w2"])
    return y + h


def decoder_block_params(hidden: int, heads: int, kv_heads: int, ffn: int, device="cuda", seed: int = 0, dtype=torch.float32):
    """Random weights of one decoder block: QKV for ``heads`` query and ``kv_heads`` key and value heads, their norms' gains,
    projection, gated feed-forward of width ``ffn``, two LayerNorms."""
    g = torch.Generator(device=device).manual_seed(seed)
    dim = hidden // heads

    def mat(rows, cols):
        return torch.nn.Parameter((torch.randn(rows, cols, generator=g, device=device) * 0.03).to(dtype))

    def vec(size, value):
        return torch.nn.Parameter(torch.full((size,), value, device=device))

    return {"wqkv": mat((heads + 2 * kv_heads) * dim, hidden), "wo": mat(hidden, hidden), "w1": mat(2 * ffn, hidden), "w2": mat(hidden, ffn),
            "gq": vec(dim, 1.0), "gk": vec(dim, 1.0), "g1": vec(hidden, 1.0), "b1": vec(hidden, 0.0), "g2": vec(hidden, 1.0), "b2": vec(hidden, 0.0)}


def decoder_block(x: torch.Tensor, p: dict, heads: int, kv_heads: int, table, position_ids=None, keep_ppm: int = 100000, bits: int = 8,
                  block: int = 64, act: int = sf.ACT_SILU, recompute: bool = False, lengths=None, bias_table=None, bucket_of=None) -> torch.Tensor:
    """One pre-LN decoder block (causal attention, queries and keys normed and turned, gated feed-forward) with the compressed
    caches of this module.  Whether a layer is frozen is read off its weight: a frozen one keeps nothing of its input (a
    LayerNorm the ``keep_ppm`` largest entries), an active one forms its weight gradient from its ``bits``-bit cache.  A place
    outside of ``table`` leaves a token unturned, not unseen: padding has to come after the tokens that count.  ``recompute`` keeps
    no probabilities, and is bound to no number of tokens: attention forms them again, and takes the sequences' ``lengths`` and a
    position bias (AttentionFunction)."""
    if not recompute:
        _only_recomputed(lengths, bias_table, bucket_of)
    B, T, H = x.shape
    D, group = H // heads, heads // kv_heads

    def norm(t, gamma, beta):
        frozen = not gamma.requires_grad
        return LayerNormFunction.apply(t, gamma, beta, 1e-5, frozen, keep_ppm, 0 if frozen else bits, block)

    qkv = LinearFunction.apply(norm(x, p["g1"], p["b1"]), p["wqkv"], None, bits, block, True)
    # a cache's blocks lie in one head; heads that have no whole block keep the rows themselves
    q, kt, v = HeadsNormRotateFunction.apply(qkv, p["gq"], p["gk"], heads, kv_heads, table, sf.ROTARY_HALVES, position_ids, 1.0 / D ** 0.5, 1e-6,
                                             bits if D % 32 == 0 else 0, block if D % block == 0 else 32)
    if recompute:
        a = AttentionFunction.apply(q, kt, v, 1.0, True, lengths, bias_table, bucket_of, sf.HEADS_APART).view(B, T, H)
    else:
        s = MatmulFunction.apply(q.view(B, kv_heads, group * T, D), kt, bits, block)       # heads that share keys are rows of one product
        later = torch.ones(T, T, dtype=torch.bool, device=x.device).triu(1)
        s = s.view(B, kv_heads, group, T, T).masked_fill(later, -1e30).view(B, kv_heads, group * T, T)
        a = SoftmaxMatmulFunction.apply(s, v, keep_ppm, bits, block).view(B, heads, T, D).transpose(1, 2).reshape(B, T, H)
    y = x + LinearFunction.apply(a, p["wo"], None, bits, block, True)
    h = LinearFunction.apply(norm(y, p["g2"], p["b2"]), p["w1"], None, bits, block, True)
    return y + LinearFunction.apply(GatedFunction.apply(h, act, bits, block), p["w2"], None, bits, block, True)


def held_activation_bytes(fn) -> tuple:
    """(bytes that stay allocated between the forward pass of ``fn`` and its backward pass, apart from the output;
    milliseconds of forward + backward)."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = torch.cuda.memory_allocated()
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    out = fn()
    torch.cuda.synchronize()
    kept = torch.cuda.memory_allocated() - before - out.numel() * out.element_size()
    out.sum().backward()
    t1.record()
    torch.cuda.synchronize()
    return kept, t0.elapsed_time(t1)
