// Attention forward for few queries: 32 rows a workgroup, the queries of all heads that share keys being rows (a token of a group
// of heads reads its keys once), each of the four waves a quarter of a tile of 128 keys, and the keys of a sequence shared out over
// `splits` workgroups where there are few rows in all.  The waves' sums meet in LDS, the workgroups' in memory, in order.
//
// What bounds it is the reading of keys and values: one query each of 16 sequences of 4096 tokens, 32 heads on 8 by 128, 268 MB, with the joining launch
// in 56 us, 4.8 TB/s; 64 sequences 5.8.
#pragma once

#include "attention.hpp"

namespace slimfit {
namespace {

template <typename T> constexpr int kFewStages = sizeof(T) == 2 ? 2 : 1;

// the place of a row's partial result: D sums, then the maximum and the sum they are against
__device__ __forceinline__ float *part_of(float *parts, int64_t row, int split, int splits, int dim) { return parts + (row * splits + split) * (dim + 2); }

template <typename T, int D, bool BIAS>
__global__ void __launch_bounds__(kAttnThreads, 1) few_kernel(Attention a, T *__restrict__ out, float *__restrict__ stats, float *__restrict__ parts, int blocks, int splits)
{
    constexpr int BYTES = kFewTile * kPitch<T, D>, STAGES = kFewStages<T>, APART = D + 4;
    __shared__ __align__(1024) char tiles[STAGES][2 * BYTES];
    __shared__ float tops[kAttnWaves][kOwn], totals[kAttnWaves][kOwn];
    static_assert(sizeof(tiles) >= kAttnWaves * kOwn * APART * 4, "the waves' sums meet where the tiles were");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int group = a.q_heads / a.kv_heads, rows = group * a.q_tokens, units = a.batch * a.kv_heads;
    const int unit = (int)(blockIdx.x % (unsigned)units), rest = (int)(blockIdx.x / (unsigned)units), block = rest % blocks, split = rest / blocks;
    const int batch = unit / a.kv_heads, kv = unit % a.kv_heads;
    const int first = block * kOwn, row = first + (lane & 31);                  // of the pair's rows: head of the group, then query
    const bool live = row < rows;
    const int head = kv * group + (live ? row / a.q_tokens : 0), i = live ? row % a.q_tokens : 0;
    const int keys = keys_of(a, batch);
    const int seen = live ? seen_by(a, i, keys) : 0;
    // tiles that some row of the workgroup sees, and this split's of them
    const int last = min(first + kOwn, rows) - 1, high_query = first / a.q_tokens == last / a.q_tokens ? last % a.q_tokens : a.q_tokens - 1;
    const int all = (seen_by(a, high_query, keys) + kFewTile - 1) / kFewTile;
    const int from = (int)((int64_t)all * split / splits), to = (int)((int64_t)all * (split + 1) / splits);
    const float scale = a.scale * kLog2e, by = BIAS ? kLog2e : scale;

    Own<T, D> own;
    {
        const T *const q = static_cast<const T *>(a.q.at) + batch * a.q.b + head * a.q.h + i * a.q.t;
#pragma unroll
        for (int c = 0; c < Own<T, D>::VECTORS; ++c) {
            const int n = 2 * c + half;
            own.x[c] = live && n * kPerVector<T> < a.head_dim ? *reinterpret_cast<const u32x4 *>(q + n * kPerVector<T>) : u32x4{0u, 0u, 0u, 0u};
        }
    }
    f32x16 o[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) o[n] = zeros16();
    float top = -__builtin_inff(), total = 0.0f;

    Tiles<T, D, kFewTile> kl, vl;
    kl.start(static_cast<const T *>(a.k.at) + batch * a.k.b + kv * a.k.h, a.k.t, from * kFewTile, keys, a.head_dim);
    vl.start(static_cast<const T *>(a.v.at) + batch * a.v.b + kv * a.v.h, a.v.t, from * kFewTile, keys, a.head_dim);
    auto fetch_keys = [&](int t) {
        if (t >= to) kl.left = 0;
        kl.fetch(tiles[t % STAGES]);
        kl.forward();
    };
    auto fetch_values = [&](int t) {
        if (t >= to) vl.left = 0;
        vl.fetch(tiles[t % STAGES] + BYTES);
        vl.forward();
    };
    auto land = [&](int t) {
        kl.land(tiles[t % STAGES]);
        vl.land(tiles[t % STAGES] + BYTES);
        kl.landed();
    };
    // bf16: a wave's quarter of a tile is what it has fetched itself, so that it waits for that alone, and asks for what comes two tiles on as
    // soon as the place is free.  Keys and values in turn: three more are under way behind the one it waits for.  (With a barrier for all
    // of a tile 61 us for those 56; 16 x 2048, 12 heads of 64: 26.9, 21.5.)
    constexpr bool ALONE = Tiles<T, D, kFewTile>::DIRECT;
    auto arrived = [] { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(3 * Tiles<T, D, kFewTile>::EACH) : "memory"); };
    auto read = [] { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); };
    if (from < to) {
        fetch_keys(from);
        fetch_values(from);
        if constexpr (ALONE) {
            fetch_keys(from + 1);
            fetch_values(from + 1);
            own.arrive();
        } else {
            own.arrive();
            land(from);
        }
    }
    for (int t = from; t < to; ++t) {
        const char *const tile = tiles[t % STAGES];
        const int k0 = t * kFewTile + wave * kOwn;
        if constexpr (ALONE) {
            arrived();
        } else {
            fetch_keys(t + 1);
            fetch_values(t + 1);
        }
        f32x16 s = dots<T, D>(tile, wave * kOwn, own);
        if constexpr (ALONE) {
            read();
            fetch_keys(t + 2);
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = k0 + row_of(r, half);
                const int bucket = key < seen ? a.bucket_of[key - i + a.q_tokens - 1] : -1;
                const float bias = (uint32_t)bucket < (uint32_t)a.buckets ? widened(static_cast<const T *>(a.table)[(int64_t)bucket * a.q_heads + head]) : 0.0f;
                s[r] = __builtin_fmaf(s[r], a.scale, bias);
            }
        }
        const int some = seen - k0 - 4 * half;
        float high = -__builtin_inff();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = row_of(r, 0) < some ? s[r] : -__builtin_inff();
            high = fmaxf(high, s[r]);
        }
        high = fmaxf(top, both_max(high));
        const float safe = high == -__builtin_inff() ? 0.0f : high, less = -safe * scale;
        const float down = __builtin_amdgcn_exp2f((top - safe) * by);
        top = high;
        total *= down;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[n][r] *= down;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(BIAS ? (s[r] - safe) * kLog2e : __builtin_fmaf(s[r], scale, less));
            total += s[r];
        }
        if constexpr (ALONE) {
            arrived();
            sums<T, D>(tile + BYTES, wave * kOwn, s, o);
            read();
            fetch_values(t + 2);
        } else {
            sums<T, D>(tile + BYTES, wave * kOwn, s, o);
            if (STAGES == 1) __syncthreads();
            land(t + 1);
        }
    }
    if constexpr (ALONE) kl.landed();
    // the four waves' sums
    total = both_sum(total);
    if (half == 0) {
        tops[wave][lane] = top;
        totals[wave][lane] = total;
    }
    __syncthreads();
    float high = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) high = fmaxf(high, tops[w][lane & 31]);
    const float safe = high == -__builtin_inff() ? 0.0f : high;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) sum += totals[w][lane & 31] * __builtin_amdgcn_exp2f((tops[w][lane & 31] - safe) * by);
    const float down = __builtin_amdgcn_exp2f((top - safe) * by) * (parts ? 1.0f : sum > 0.0f ? 1.0f / sum : 0.0f);
    float *const meet = reinterpret_cast<float *>(tiles[0]);
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<f32x4 *>(meet + (wave * kOwn + (lane & 31)) * APART + 32 * n + 8 * c + 4 * half) =
                f32x4{o[n][4 * c] * down, o[n][4 * c + 1] * down, o[n][4 * c + 2] * down, o[n][4 * c + 3] * down};
    if (wave == 0 && half == 0 && live) {
        if (parts) {
            float *const to_part = part_of(parts, (int64_t)unit * rows + row, split, splits, a.head_dim);
            to_part[a.head_dim] = high;
            to_part[a.head_dim + 1] = sum;
        } else {
            const int64_t at = ((int64_t)batch * a.q_heads + head) * a.q_tokens + i;
            stats[2 * at] = BIAS ? high : high * a.scale;
            stats[2 * at + 1] = sum;
        }
    }
    __syncthreads();
    const int count = min(kOwn, rows - first) * a.head_dim;
    for (int n = threadIdx.x; n < count; n += kAttnThreads) {
        const int r = n / a.head_dim, d = n % a.head_dim;
        const float *const m = meet + r * APART + d;
        const float x = ((m[0] + m[kOwn * APART]) + m[2 * kOwn * APART]) + m[3 * kOwn * APART];
        if (parts) {
            part_of(parts, (int64_t)unit * rows + first + r, split, splits, a.head_dim)[d] = x;
        } else {
            const int h = kv * group + (first + r) / a.q_tokens, q = (first + r) % a.q_tokens;
            T *const at = out + (((int64_t)batch * a.q_tokens + q) * a.q_heads + h) * a.head_dim + d;
            if constexpr (sizeof(T) == 4) *at = x;
            else *at = (T)bf16_narrow(x);
        }
    }
}

// A wave for each row: the splits' maxima and sums, one a lane, then their sums of values by lanes of D, added up in order.
template <typename T, bool BIAS>
__global__ void __launch_bounds__(kAttnThreads) few_join_kernel(Attention a, const float *__restrict__ parts, int splits, T *__restrict__ out, float *__restrict__ stats)
{
    __shared__ float weights[kAttnWaves][kMostSplits];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = a.q_heads / a.kv_heads, rows = group * a.q_tokens, apart = a.head_dim + 2;
    const int64_t row = (int64_t)blockIdx.x * kAttnWaves + wave;
    const bool live = row < (int64_t)a.batch * a.kv_heads * rows;
    const float by = BIAS ? kLog2e : a.scale * kLog2e;
    const float *const at = parts + (live ? row : 0) * splits * apart;
    const bool mine = lane < splits;
    const float top = mine ? at[lane * apart + a.head_dim] : -__builtin_inff();
    float high = top;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) high = fmaxf(high, __shfl_xor(high, o, kWave));
    const float weight = mine ? __builtin_amdgcn_exp2f((top - (high == -__builtin_inff() ? 0.0f : high)) * by) : 0.0f;
    float sum = mine ? at[lane * apart + a.head_dim + 1] * weight : 0.0f;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    weights[wave][lane] = weight;
    __syncthreads();
    if (!live) return;
    const int64_t unit = row / rows;
    const int in = (int)(row % rows), batch = (int)(unit / a.kv_heads), head = (int)(unit % a.kv_heads) * group + in / a.q_tokens, i = in % a.q_tokens;
    const float inverse = sum > 0.0f ? 1.0f / sum : 0.0f;
    T *const to = out + (((int64_t)batch * a.q_tokens + i) * a.q_heads + head) * a.head_dim;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int d = lane + 64 * n;
        if (d >= a.head_dim) continue;
        float x = 0.0f;
#pragma unroll 8
        for (int s = 0; s < splits; ++s) x += at[s * apart + d] * weights[wave][s];
        if constexpr (sizeof(T) == 4) to[d] = x * inverse;
        else to[d] = (T)bf16_narrow(x * inverse);
    }
    if (lane == 0) {
        const int64_t place = ((int64_t)batch * a.q_heads + head) * a.q_tokens + i;
        stats[2 * place] = BIAS ? high : high * a.scale;
        stats[2 * place + 1] = sum;
    }
}

template <typename T, int D>
void launch_few(const Attention &a, T *out, float *stats, float *parts, int splits, hipStream_t st)
{
    const int group = a.q_heads / a.kv_heads, rows = group * a.q_tokens, blocks = (rows + kOwn - 1) / kOwn;
    const unsigned grid = (unsigned)((int64_t)a.batch * a.kv_heads * blocks * splits);
    float *const to = splits > 1 ? parts : nullptr;
    if (a.table) launch(few_kernel<T, D, true>, grid, kAttnThreads, 0, st, a, out, stats, to, blocks, splits);
    else launch(few_kernel<T, D, false>, grid, kAttnThreads, 0, st, a, out, stats, to, blocks, splits);
    if (splits == 1) return;
    const unsigned joins = (unsigned)(((int64_t)a.batch * a.kv_heads * rows + kAttnWaves - 1) / kAttnWaves);
    if (a.table) launch(few_join_kernel<T, true>, joins, kAttnThreads, 0, st, a, parts, splits, out, stats);
    else launch(few_join_kernel<T, false>, joins, kAttnThreads, 0, st, a, parts, splits, out, stats);
}

}  // namespace
}  // namespace slimfit
