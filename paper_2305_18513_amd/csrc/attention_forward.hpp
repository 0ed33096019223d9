// Attention forward, one pass over the keys:  s = scale q k^T + bias, m = max s, l = sum e^(s - m), out = sum e^(s - m) v / l.
// A workgroup holds 128 queries of one head, 32 a wave, and goes over tiles of 64 keys and values; maximum, sum and out are kept as
// they are so far, and taken down by e^(old - new maximum) where a tile raises the maximum.  (s^T lies with a query in each lane, so
// that the maximum and sum are a lane's own, but for one exchange of the halves.)
//
// What bounds it: bf16, the exponentials and what else is done to each of s (vector instructions 42 to 56 % of the time, matrix instructions 30 to
// 42 %); fp32, matrix instructions.  8 x 2048, 32 heads of 128 on 8: 621 us (0.89 PFLOP/s); 16 x 1024, 16 heads of 64: 93 (0.74); fp32, 2 x 4096, 16 heads of
// 64: 1070 (129 TFLOP/s).
#pragma once

#include "attention_few.hpp"

namespace slimfit {
namespace {

template <typename T, int D, bool BIAS>
__global__ void __launch_bounds__(kAttnThreads, sizeof(T) == 4 && D > 64 ? 1 : 2) forward_kernel(Attention a, T *__restrict__ out, float *__restrict__ stats, int blocks)
{
    __shared__ __align__(1024) char keys_lds[2][kTileBytes<T, D>], values_lds[2][kTileBytes<T, D>];
    __shared__ float column[BIAS ? kMostBuckets : 1], biases[2][BIAS ? kDistances : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int group = a.q_heads / a.kv_heads;
    const Place place(a.batch * a.kv_heads, blocks, group, a.causal != 0);
    const int block = a.causal ? blocks - 1 - place.block : place.block;       // the longest first
    const int batch = place.unit / a.kv_heads, kv = place.unit % a.kv_heads, head = kv * group + place.in, bh = batch * a.q_heads + head;
    const int q0 = block * kBlock, mine = q0 + wave * kOwn, i = mine + (lane & 31);
    const T *const q = static_cast<const T *>(a.q.at) + batch * a.q.b + head * a.q.h;
    const T *const k = static_cast<const T *>(a.k.at) + batch * a.k.b + kv * a.k.h;
    const T *const v = static_cast<const T *>(a.v.at) + batch * a.v.b + kv * a.v.h;
    const int keys = keys_of(a, batch), count = key_tiles(a, q0, keys);
    const int seen = seen_by(a, i, keys), all_see = seen_by(a, mine, keys), any_sees = mine < a.q_tokens ? seen_by(a, min(mine + kOwn, a.q_tokens) - 1, keys) : 0;
    const float scale = a.scale * kLog2e;

    Own<T, D> own;
    own.load(q, a.q.t, mine, a.q_tokens, a.head_dim);
    f32x16 o[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = zeros16();
    // Of q k^T, or (BIAS) of s: the maximum so far, and what the exponentials are taken against.  That follows only where the maximum has
    // risen by 2^8 and more: e^(s - base) and its sums have room for that, and out is rarely taken down.
    float top = -__builtin_inff(), base = -__builtin_inff(), total = 0.0f;
    // (A finite room, also for the least scales: -infinity and an infinite one would be none.)
    const float by = BIAS ? kLog2e : scale, room = fminf(8.0f / by, 0x1.fffffep127f);

    Tiles<T, D> kl, vl;
    BiasLoad bl;
    kl.start(k, a.k.t, 0, keys, a.head_dim);
    vl.start(v, a.v.t, 0, keys, a.head_dim);
    auto fetch_keys = [&](int t) { kl.fetch(keys_lds[t & 1]); kl.forward(); };
    auto fetch_values = [&](int t) { vl.fetch(values_lds[t & 1]); vl.forward(); };
    auto fetch_bias = [&](int t) { if constexpr (BIAS) bl.load(a, t * kTile - q0 - (kBlock - 1) + a.q_tokens - 1); };
    auto land_bias = [&](int t) { if constexpr (BIAS) bl.store(a, column, biases[t & 1]); };

    // A tile's products with the queries are formed while the exponentials of the one before it are: keys are a tile ahead of values.
    f32x16 s[2][2];
    if (count > 0) {
        if constexpr (BIAS) load_column<T>(a, head, column);
        fetch_keys(0);
        kl.land(keys_lds[0]);
        fetch_keys(1);
        kl.land(keys_lds[1]);
        fetch_values(0);
        vl.land(values_lds[0]);
        fetch_bias(0);
        own.arrive();
        if constexpr (BIAS) {
            __syncthreads();
            land_bias(0);
        }
        kl.landed();
        dots2<T, D>(keys_lds[0], own, s[0], (any_sees + 31) / 32);
        __syncthreads();
    }
    auto step = [&](int t, f32x16 (&s)[2], f32x16 (&next)[2]) {
        const int k0 = t * kTile;
        fetch_keys(t + 2);
        fetch_values(t + 1);
        fetch_bias(t + 1);
        if (k0 < any_sees) {
            if constexpr (BIAS) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float *const b = biases[t & 1] + kBlock - 1 - (i - q0) + 4 * half + 32 * n;
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[n][r] = __builtin_fmaf(s[n][r], a.scale, b[8 * (r / 4) + r % 4]);
                }
            }
            if (k0 + kTile > all_see) {
                const int count = seen - k0 - 4 * half;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[n][r] = 32 * n + row_of(r, 0) < count ? s[n][r] : -__builtin_inff();
            }
            float high = s[0][0];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) high = fmaxf(high, s[n][r]);
            top = fmaxf(top, both_max(high));
            if (__builtin_amdgcn_ballot_w64(top > base + room) != 0u) {
                const float down = __builtin_amdgcn_exp2f((base - (top == -__builtin_inff() ? 0.0f : top)) * by);     // (no key so far: 0 of 0)
                total *= down;
#pragma unroll
                for (int n = 0; n < D / 32; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[n][r] *= down;
                base = top;
            }
            const float safe = base == -__builtin_inff() ? 0.0f : base, less = -safe * scale;
            dots2<T, D>(keys_lds[(t + 1) & 1], own, next, (any_sees - k0 - kTile + 31) / 32);           // (past the last tile: of keys that are not there, unused)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    // (with a bias s may be the type's lowest value, which times log2 e is none: the difference comes first)
                    s[n][r] = __builtin_amdgcn_exp2f(BIAS ? (s[n][r] - safe) * kLog2e : __builtin_fmaf(s[n][r], scale, less));
                    total += s[n][r];
                }
                if (sizeof(T) == 2 || k0 + 32 * n < any_sees) sums<T, D>(values_lds[t & 1], 32 * n, s[n], o);
            }
            if constexpr (sizeof(T) == 2) {                 // products, reads and exponentials in turn: 402 us without, 373 with (8 x 2048 x 2048 by 128 causal, 32 heads on 8)
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                for (int x = 0; x < D / 8; ++x) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x400, 128 / D, 0);
                }
#pragma unroll
                for (int x = 0; x < D / 8; ++x) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);
                    __builtin_amdgcn_sched_group_barrier(0x400, 128 / D, 0);
                }
            }
        }
        kl.land(keys_lds[t & 1]);
        vl.land(values_lds[(t + 1) & 1]);
        land_bias(t + 1);
        kl.landed();
    };
    for (int t = 0; t < count; t += 2) {
        step(t, s[0], s[1]);
        if (t + 1 < count) step(t + 1, s[1], s[0]);
    }
    total = both_sum(total);
    const float inverse = total > 0.0f ? 1.0f / total : 0.0f;
    if (total > 0.0f) total *= __builtin_amdgcn_exp2f((base - top) * by);       // against the maximum itself, for the backward pass
    if (i < a.q_tokens) {
        const int64_t row = ((int64_t)batch * a.q_tokens + i) * a.q_heads + head;
        store_row<T, D>(o, inverse, out + row * a.head_dim, a.head_dim);
        if (half == 0) {
            const int64_t at = (int64_t)bh * a.q_tokens + i;
            stats[2 * at] = BIAS ? top : top * a.scale;
            stats[2 * at + 1] = total;
        }
    }
}

template <typename T, int D>
void launch_forward(const Attention &a, T *out, float *stats, hipStream_t st)
{
    const int blocks = (a.q_tokens + kBlock - 1) / kBlock;
    const unsigned grid = (unsigned)((int64_t)a.batch * a.q_heads * blocks);
    if (a.table) launch(forward_kernel<T, D, true>, grid, kAttnThreads, 0, st, a, out, stats, blocks);
    else launch(forward_kernel<T, D, false>, grid, kAttnThreads, 0, st, a, out, stats, blocks);
}

template <typename T, int D>
void launch_either(const Attention &a, T *out, float *stats, float *parts, int splits, hipStream_t st)
{
    if (splits > 0) launch_few<T, D>(a, out, stats, parts, splits, st);
    else launch_forward<T, D>(a, out, stats, st);
}

template <typename T>
void attention_forward_of(const Attention &a, void *out, float *stats, float *parts, int splits, hipStream_t st)
{
    T *o = static_cast<T *>(out);
    if (a.head_dim <= 32) launch_either<T, 32>(a, o, stats, parts, splits, st);
    else if (a.head_dim <= 64) launch_either<T, 64>(a, o, stats, parts, splits, st);
    else if (a.head_dim <= 96) launch_either<T, 96>(a, o, stats, parts, splits, st);
    else launch_either<T, 128>(a, o, stats, parts, splits, st);
}

}  // namespace
}  // namespace slimfit
