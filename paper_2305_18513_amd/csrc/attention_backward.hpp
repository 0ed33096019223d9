// Attention backward from recomputed probabilities:  p = e^(s - m) / l,  dp = dout v^T,  delta = sum over d of dout out,  ds = p (dp - delta),
//     dq = scale ds k,   dk = scale ds^T q,   dv = p^T dout,   dtable[b] = sum of ds over the pairs of bucket b.
// Two kernels, so that every sum has one owner and one order: a wave of the first holds 32 queries and goes over keys (dq, and the
// sums of ds by distance), a wave of the second 32 keys and goes over the queries of all heads that share them (dk, dv).  They form s
// and dp twice: seven products where five would do with sums that meet in memory.
//
// What bounds them: bf16, vector instructions (exponentials at a quarter of the rate) and matrix instructions, 35 to 50 % of the time each,
// of which two waves a SIMD, as many as the registers allow, overlap a part; fp32, matrix instructions.  8 x 2048, 32 heads of 128 on 8: queries
// 802 us (1.0 PFLOP/s of its three products), keys 1474 (0.75 of its four); 16 x 1024, 16 heads of 64: 150 (0.92, four with p k) and 179 (0.77); fp32, 2 x
// 4096, 16 heads of 64: 1540 (134 TFLOP/s) and 1970 (139).  (Keys' s and dp of 32 queries ahead of the exponentials of the 32
// before, in three stages of tiles: 121 us where this takes 119, 1024 x 1024 by 64 causal and 256 heads.)
#pragma once

#include "attention.hpp"

#include <type_traits>

namespace slimfit {
namespace {

// p = exp2(fma(q k^T, scale log2 e, -first)), or with a bias exp2((s - first) log2 e - second).  A query that sees no key has first
// or second infinite, its p are 0.
template <bool BIAS> __device__ __forceinline__ float probability(float s, float scale, float first, float second)
{
    return __builtin_amdgcn_exp2f(BIAS ? __builtin_fmaf(s - first, kLog2e, -second) : __builtin_fmaf(s, scale, -first));
}

constexpr int kSkew = kOwn + 4;              // floats of a query's ds in LDS

// delta from an out that was rounded to bf16 is off by e = sum of dout (out - rounded), and ds by e p: more than ds's own rounding where a
// query sees few keys, or one key takes most of it.  The sum of a query's ds is -e, as it should be nothing.  Heads of up to 96
// form sum of p k beside dq and take e of it off at the end (1024 x 1024 by 64 causal, 256 heads: 81 us without, 98 with; dq's error
// against 64 bits goes from 2.1 times that of one rounding of the result to 1.4, at inputs with a thousandth of outliers).  Heads of 128 have no
// registers left for that (469 us without, 702 with the rows of dout in LDS): theirs go over the keys twice where these are no
// more than kTwiceTiles tiles, or one takes more than half of some query's p (a sum of exponentials below 2: in a seventh to a fourth of the
// blocks at such inputs, and dq's error 1.4 roundings again), once for delta = sum of p dp.  So do those with a bias, at any length: sums of ds over a bucket of many keys are
// little but e otherwise (two buckets: 5 % off), and whether the table takes a gradient changes no other.  Keys' gradients take
// the right delta in any case.
template <typename T, int D, bool ALWAYS> constexpr bool kRights = sizeof(T) == 2 && D <= 96 && !ALWAYS;
template <typename T, int D, bool ALWAYS> constexpr bool kTwice = sizeof(T) == 2 && !kRights<T, D, ALWAYS>;
constexpr int kTwiceTiles = 2;

template <typename T, int D, bool BIAS, bool PARTS, bool SPLIT>
__global__ void __launch_bounds__(kAttnThreads, D * sizeof(T) > (PARTS ? 128 : 256) ? 1 : 2) queries_kernel(Attention a, Gradients g, int blocks)
{
    __shared__ __align__(1024) char tiles[2][2 * kTileBytes<T, D>];
    __shared__ float column[BIAS ? kMostBuckets : 1], biases[2][BIAS ? kDistances : 1];
    __shared__ __align__(16) float skew[PARTS ? kAttnWaves : 1][PARTS ? kOwn * kSkew : 1];
    __shared__ int buckets[2][PARTS ? kDistances : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int group = a.q_heads / a.kv_heads;
    const int splits = SPLIT ? g.q_splits : 1;
    const Place place(a.batch * a.kv_heads, blocks * splits, group, a.causal != 0);
    const int at_block = a.causal ? blocks - 1 - place.block / splits : place.block / splits, split = place.block % splits;     // the longest first
    const int block = PARTS ? g.first_block + at_block : at_block;
    const int batch = place.unit / a.kv_heads, kv = place.unit % a.kv_heads, head = kv * group + place.in, bh = batch * a.q_heads + head;
    const int q0 = block * kBlock, mine = q0 + wave * kOwn, i = mine + (lane & 31);
    const T *const q = static_cast<const T *>(a.q.at) + batch * a.q.b + head * a.q.h;
    const T *const k = static_cast<const T *>(a.k.at) + batch * a.k.b + kv * a.k.h;
    const T *const v = static_cast<const T *>(a.v.at) + batch * a.v.b + kv * a.v.h;
    const int keys = keys_of(a, batch), all_tiles = key_tiles(a, q0, keys);
    const int t0 = SPLIT ? first_of(all_tiles, split, splits) : 0, count = SPLIT ? first_of(all_tiles, split + 1, splits) : all_tiles;
    const int seen = seen_by(a, i, keys), all_see = seen_by(a, mine, keys), any_sees = mine < a.q_tokens ? seen_by(a, min(mine + kOwn, a.q_tokens) - 1, keys) : 0;
    const float scale = a.scale * kLog2e;
    constexpr bool ALWAYS = BIAS || SPLIT;                  // goes over the keys twice at any length
    // (where tiles are shared out each goes over all of them for delta: from tile `start` to `end` first)
    bool twice = kTwice<T, D, ALWAYS> && (ALWAYS ? !SPLIT || split == 0 || count > t0 : all_tiles <= kTwiceTiles), wave_twice = true;
    if constexpr (kTwice<T, D, ALWAYS> && !ALWAYS) {
        __shared__ int one_takes_most[kAttnWaves];
        const float total = i < a.q_tokens ? g.stats[2 * ((int64_t)bh * a.q_tokens + i) + 1] : 0.0f;
        wave_twice = twice || __builtin_amdgcn_ballot_w64(total > 0.0f && total < 2.0f) != 0u;      // (the largest of e^(s - m) is 1)
        if (lane == 0) one_takes_most[wave] = wave_twice;
        __syncthreads();
        twice = (one_takes_most[0] | one_takes_most[1] | one_takes_most[2] | one_takes_most[3]) != 0;
    }
    const int start = twice ? 0 : t0, end = twice ? all_tiles : count;

    Tiles<T, D> kl, vl;
    BiasLoad bl;
    kl.start(k, a.k.t, start * kTile, keys, a.head_dim);
    vl.start(v, a.v.t, start * kTile, keys, a.head_dim);
    auto fetch = [&](int t) {
        kl.fetch(tiles[t & 1]);
        vl.fetch(tiles[t & 1] + kTileBytes<T, D>);
        kl.forward();
        vl.forward();
        if constexpr (BIAS) bl.load(a, t * kTile - q0 - (kBlock - 1) + a.q_tokens - 1);
    };
    auto land = [&](int t) {
        kl.land(tiles[t & 1]);
        vl.land(tiles[t & 1] + kTileBytes<T, D>);
        if constexpr (BIAS) bl.store(a, column, biases[t & 1]);
        if constexpr (PARTS)
            if (threadIdx.x < kDistances) buckets[t & 1][threadIdx.x] = bl.bucket;
        kl.landed();
    };

    Own<T, D> own, grad;
    own.load(q, a.q.t, mine, a.q_tokens, a.head_dim);
    const int64_t out_row = (int64_t)a.q_heads * a.head_dim, out_at = (int64_t)batch * a.q_tokens * out_row + (int64_t)head * a.head_dim;
    grad.load(static_cast<const T *>(g.dout) + out_at, out_row, mine, a.q_tokens, a.head_dim);
    float first = __builtin_inff(), second = __builtin_inff(), delta = 0.0f;
    {
        Own<T, D> o;
        o.load(static_cast<const T *>(g.out) + out_at, out_row, mine, a.q_tokens, a.head_dim);
#pragma unroll
        for (int c = 0; c < Own<T, D>::VECTORS; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t x = o.x[c][e], y = grad.x[c][e];
                if constexpr (sizeof(T) == 4) {
                    delta = __builtin_fmaf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y), delta);
                } else {
                    delta = __builtin_fmaf(__builtin_bit_cast(float, x << 16), __builtin_bit_cast(float, y << 16), delta);
                    delta = __builtin_fmaf(__builtin_bit_cast(float, x & 0xFFFF0000u), __builtin_bit_cast(float, y & 0xFFFF0000u), delta);
                }
            }
        delta = both_sum(delta);
    }
    if (i < a.q_tokens) {
        const int64_t at = (int64_t)bh * a.q_tokens + i, all = (int64_t)a.batch * a.q_heads * a.q_tokens;
        const float top = g.stats[2 * at], total = g.stats[2 * at + 1];
        if (!(total <= 0.0f)) {                             // (a sum of NaN too: its p are NaN)
            const float l = __builtin_amdgcn_logf(total);   // to the base of 2
            first = BIAS ? top : __builtin_fmaf(top, kLog2e, l);
            second = l;
        } else if (BIAS) {
            first = 0.0f;                                   // (second stays infinite)
        }
        if (half == 0 && split == 0) {                      // for the second kernel
            g.rows[at] = first;
            g.rows[all + at] = second;
        }
    }
    f32x16 dq[D / 32], pk[kRights<T, D, ALWAYS> ? D / 32 : 1];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) {
        dq[n] = zeros16();
        if constexpr (kRights<T, D, ALWAYS>) pk[n] = zeros16();
    }
    float off = 0.0f;                                       // -e
    float carry = 0.0f;
    float *const part = PARTS ? g.parts + (((int64_t)bh * blocks + at_block) * splits + split) * kAttnWaves * g.part_row + wave * g.part_row : nullptr;

    if constexpr (BIAS) {
        load_column<T>(a, head, column);
        __syncthreads();
    }
    // p and dp of 32 keys, p of those that a query does not see left as it is; and whether there are any
    auto pairs = [&](int t, int n, f32x16 &p, f32x16 &dp) {
        const char *const tile = tiles[t & 1];
        p = dots<T, D>(tile, 32 * n, own);
        dp = dots<T, D>(tile + kTileBytes<T, D>, 32 * n, grad);
        const float *const b = biases[BIAS ? t & 1 : 0] + kBlock - 1 - (i - q0) + 4 * half + 32 * n;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if constexpr (BIAS) p[r] = __builtin_fmaf(p[r], a.scale, b[8 * (r / 4) + r % 4]);
            p[r] = probability<BIAS>(p[r], scale, first, second);
        }
        return t * kTile + 32 * n + 32 > all_see;
    };
    auto leave_out = [&](int t, int n, f32x16 &x) {
        const int some = seen - t * kTile - 32 * n - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = row_of(r, 0) < some ? x[r] : 0.0f;
    };
    if (end > start) {
        fetch(start);
        own.arrive();
        grad.arrive();
        land(start);
    }
    if (twice) {
        float x = 0.0f, y = 0.0f;
        for (int t = start; t < end; ++t) {
            fetch(t + 1);
            if (wave_twice && t * kTile < any_sees)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    f32x16 p, dp;
                    if (pairs(t, n, p, dp)) {
                        leave_out(t, n, p);
                        leave_out(t, n, dp);
                    }
#pragma unroll
                    for (int r = 0; r < 16; r += 2) {
                        x = __builtin_fmaf(p[r], dp[r], x);
                        y = __builtin_fmaf(p[r + 1], dp[r + 1], y);
                    }
                }
            land(t + 1);
        }
        if (wave_twice) delta = both_sum(x + y);
        if (count > t0) {
            kl.start(k, a.k.t, t0 * kTile, keys, a.head_dim);
            vl.start(v, a.v.t, t0 * kTile, keys, a.head_dim);
            fetch(t0);
            land(t0);
        }
    }
    for (int t = t0; t < count; ++t) {
        const char *const tile = tiles[t & 1];
        const int k0 = t * kTile;
        fetch(t + 1);
        if (k0 < any_sees) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                // (products are what takes fp32's time; with the sums by distance every half is gone through)
                if (sizeof(T) == 4 && !PARTS && k0 + 32 * n >= any_sees) continue;
                f32x16 p, s;
                const bool some = pairs(t, n, p, s);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = p[r] * (s[r] - delta);
                if (some) {
                    leave_out(t, n, s);
                    if constexpr (kRights<T, D, ALWAYS>) leave_out(t, n, p);
                }
                if constexpr (sizeof(T) == 2 && !ALWAYS) {
                    float x = s[0], y = s[1];
#pragma unroll
                    for (int r = 2; r < 16; r += 2) {
                        x += s[r];
                        y += s[r + 1];
                    }
                    off += x + y;
                }
                if constexpr (PARTS) {
                    // Sums by distance, key - query.  Within 32 keys and the wave's 32 queries lane l has those of l - 31 (lower) and of l + 1
                    // (upper), which the next 32 keys see 32 lower.  Where all 63 are of one bucket, as far ones are, their sum goes to one of them.
                    const int *const b = buckets[t & 1] + kBlock - kOwn - wave * kOwn + 32 * n;
                    const int mine_of = b[min(lane, 62)];
                    float lower = 0.0f, upper = 0.0f;
                    if (__builtin_amdgcn_ballot_w64(mine_of != __builtin_amdgcn_readfirstlane(mine_of)) == 0u) {
                        float x[16];
#pragma unroll
                        for (int r = 0; r < 16; ++r) x[r] = s[r];
#pragma unroll
                        for (int w = 8; w >= 1; w >>= 1)
#pragma unroll
                            for (int r = 0; r < w; ++r) x[r] += x[r + w];
                        const float all_of = group_sum_f32(x[0], kWave);
                        lower = lane == 0 ? all_of : 0.0f;
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            *reinterpret_cast<f32x4 *>(&skew[wave][(lane & 31) * kSkew + 8 * c + 4 * half]) = f32x4{s[4 * c], s[4 * c + 1], s[4 * c + 2], s[4 * c + 3]};
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        __builtin_amdgcn_wave_barrier();
#pragma unroll
                        for (int m = 0; m < kOwn / 2; ++m) {                  // half of the queries each half of the wave
                            const int query = 16 * half + m, key = (lane & 31) + query + 1;
                            const float x = skew[wave][query * kSkew + (key & 31)];
                            upper += key < 32 ? x : 0.0f;
                            lower += key < 32 ? 0.0f : x;
                        }
                        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        lower = both_sum(lower);
                        upper = both_sum(upper);
                    }
                    if (half == 0) part[k0 - t0 * kTile + 32 * n + lane] = lower + carry;
                    carry = upper;
                }
                if constexpr (kRights<T, D, ALWAYS>) sums_of_two<D>(tile, 32 * n, s, dq, p, pk);
                else sums<T, D>(tile, 32 * n, s, dq);
            }
        } else if (PARTS) {
            part[k0 - t0 * kTile + lane] = half == 0 ? carry : 0.0f;
            carry = 0.0f;
        }
        land(t + 1);
    }
    if (PARTS && half == 0) part[(count - t0) * kTile + lane] = carry;
    if constexpr (sizeof(T) == 2 && !ALWAYS) off = both_sum(off);
    if constexpr (kRights<T, D, ALWAYS>) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[n][r] = __builtin_fmaf(-off, pk[n][r], dq[n][r]);
    }
    if (half == 0 && split == 0 && i < a.q_tokens) g.rows[2 * (int64_t)a.batch * a.q_heads * a.q_tokens + (int64_t)bh * a.q_tokens + i] = delta + off;      // for the second kernel
    if (SPLIT) {
        if (i < a.q_tokens)
            store_row<float, D>(dq, a.scale, g.dq_parts + (((int64_t)split * a.batch * a.q_heads + bh) * a.q_tokens + i) * a.head_dim, a.head_dim);
        return;
    }
    if (i < a.q_tokens) store_row<T, D>(dq, a.scale, static_cast<T *>(g.dq) + batch * g.dq_b + head * g.dq_h + i * g.dq_t, a.head_dim);
}

// bf16 heads of 96 and 128: two waves a SIMD have no room for all of the wave's own rows, of which the values stay in LDS, with smaller
// tiles to make up for them.
template <typename T, int D> constexpr bool kValuesInLds = sizeof(T) == 2 && D > 64;

// (fp32 heads of 64 with a bias: two waves a SIMD keep 68 registers in memory, 165 us for one wave's 178, 8 x 512, 12 heads; where blocks are
// shared out there is one workgroup a compute unit anyway, 36 and 31, 2 x 300.  Of the other kernels for two waves bf16 heads of 128 with a bias keep 20 to 23
// there; those of 64 with a bias, of 96, and of 128 without, up to 5, fp32 ones of 64 one.)
template <typename T, int D, bool BIAS, bool SPLIT>
__global__ void __launch_bounds__(kAttnThreads, sizeof(T) == 4 && D > (BIAS && SPLIT ? 32 : 64) ? 1 : 2) keys_kernel(Attention a, Gradients g, int blocks)
{
    constexpr int ROWS = kValuesInLds<T, D> ? 32 : kTile, BYTES = ROWS * kPitch<T, D>;
    __shared__ __align__(1024) char tiles[2][2 * BYTES], values[kValuesInLds<T, D> ? kBlock * kPitch<T, D> : 16];
    __shared__ __align__(16) float rows[2][3][ROWS];
    __shared__ float column[BIAS ? kMostBuckets : 1], biases[2][BIAS ? kDistances : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int splits = SPLIT ? g.k_splits : 1;
    const Place place(a.batch * a.kv_heads, blocks * splits, 1, a.causal != 0);
    const int batch = place.unit / a.kv_heads, kv = place.unit % a.kv_heads, block = place.block / splits, split = place.block % splits, group = a.q_heads / a.kv_heads;
    const int k0 = block * kBlock, mine = k0 + wave * kOwn, j = mine + (lane & 31);
    const int keys = keys_of(a, batch);
    const float scale = a.scale * kLog2e;
    const int64_t out_row = (int64_t)a.q_heads * a.head_dim, all = (int64_t)a.batch * a.q_heads * a.q_tokens;

    // queries that see the first of the workgroup's keys, and all of the wave's
    const int offset = a.k_tokens - a.q_tokens;
    const int from = a.causal ? max(0, k0 - offset) / ROWS : 0, per_head = k0 < keys ? max(0, (a.q_tokens + ROWS - 1) / ROWS - from) : 0;
    const int all_tiles = per_head * group, t0 = SPLIT ? first_of(all_tiles, split, splits) : 0, count = SPLIT ? first_of(all_tiles, split + 1, splits) : all_tiles;

    Own<T, D> own;
    Own<T, kValuesInLds<T, D> ? 32 : D> val;
    own.load(static_cast<const T *>(a.k.at) + batch * a.k.b + kv * a.k.h, a.k.t, mine, keys, a.head_dim);
    const T *const v = static_cast<const T *>(a.v.at) + batch * a.v.b + kv * a.v.h;
    if constexpr (!kValuesInLds<T, D>) val.load(v, a.v.t, mine, keys, a.head_dim);
    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = zeros16();

    Tiles<T, D, ROWS> ql, gl;
    BiasLoad bl;
    float held[3];
    // Tiles of queries from the last to the first, of each the heads in turn, so that the workgroups of a pair read the same ones at
    // about the same time, whatever their keys' place.
    int q0 = (from + per_head - 1 - t0 / group) * ROWS, next = t0 % group;     // where `fetch` stands: the tile's first query, the head of the group
    ql.start(static_cast<const T *>(a.q.at) + batch * a.q.b + (kv * group + next) * a.q.h, a.q.t, q0, a.q_tokens, a.head_dim);
    gl.start(static_cast<const T *>(g.dout) + (int64_t)batch * a.q_tokens * out_row + (int64_t)(kv * group + next) * a.head_dim, out_row, q0, a.q_tokens, a.head_dim);
    const int64_t q_head = a.q.h * (int64_t)sizeof(T), out_head = a.head_dim * (int64_t)sizeof(T);
    const float *row_at = g.rows + ((int64_t)batch * a.q_heads + kv * group + next) * a.q_tokens + q0 + (int64_t)threadIdx.x;
    auto fetch = [&](int t) {
        ql.fetch(tiles[t & 1]);
        gl.fetch(tiles[t & 1] + BYTES);
        const bool in = threadIdx.x < ROWS && q0 + (int)threadIdx.x < a.q_tokens && t < count;
        held[0] = in ? row_at[0] : BIAS ? 0.0f : __builtin_inff();
        held[1] = BIAS && in ? row_at[all] : __builtin_inff();
        held[2] = in ? row_at[2 * all] : 0.0f;
        if constexpr (BIAS) bl.load(a, k0 - q0 - (ROWS - 1) + a.q_tokens - 1);
        if (++next < group) {
            ql.at += q_head;
            gl.at += out_head;
            row_at += a.q_tokens;
        } else {
            next = 0;
            q0 -= ROWS;
            ql.at -= (group - 1) * q_head + ql.step;
            gl.at -= (group - 1) * out_head + gl.step;
            row_at -= (int64_t)(group - 1) * a.q_tokens + ROWS;
            ql.left = t + 1 < count ? ql.left + ql.step : 0;
            gl.left = t + 1 < count ? gl.left + gl.step : 0;
        }
    };
    auto land = [&](int t) {
        ql.land(tiles[t & 1]);
        gl.land(tiles[t & 1] + BYTES);
        if (threadIdx.x < ROWS) {
#pragma unroll
            for (int n = 0; n < 3; ++n) rows[t & 1][n][threadIdx.x] = held[n];
        }
        if constexpr (BIAS) bl.store(a, column, biases[t & 1]);
        ql.landed();
    };
    if (count > t0) {
        if constexpr (BIAS) {
            load_column<T>(a, kv * group + t0 % group, column);
            __syncthreads();
        }
        fetch(t0);
        if constexpr (kValuesInLds<T, D>) {
            Tiles<T, D, kBlock> vl;
            vl.start(v, a.v.t, k0, keys, a.head_dim);
            vl.fetch(values);
        } else {
            val.arrive();
        }
        own.arrive();
        land(t0);
    }
    // the first query that sees the lane's key
    const int visible = j >= keys ? 0x7FFFFFFF : a.causal ? j - offset : -0x7FFFFFFF;
    for (int t = t0; t < count; ++t) {
        const char *const tile = tiles[t & 1];
        const int here = (from + per_head - 1 - t / group) * ROWS;
        fetch(t + 1);
#pragma unroll
        for (int n = 0; n < ROWS / 32; ++n) {
            const int first = here + 32 * n;                // of 32 queries
            // none of them sees any of the wave's keys, or none is there (products are what takes fp32's time)
            if (sizeof(T) == 4 && (mine >= keys || first >= a.q_tokens || (a.causal && first + 31 + offset < mine))) continue;
            f32x16 s = dots<T, D>(tile, 32 * n, own);
            f32x16 dp;
            if constexpr (kValuesInLds<T, D>) dp = dots_of<T, D>(tile + BYTES, 32 * n, values + wave * kOwn * kPitch<T, D>);
            else dp = dots<T, D>(tile + BYTES, 32 * n, val);
            const float *const b = biases[BIAS ? t & 1 : 0] + ROWS - 1 + (j - k0) - 32 * n - 4 * half;
            const int none = visible > first + 64 ? 64 : visible < first ? 0 : visible - first;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4 f = *reinterpret_cast<const f32x4 *>(&rows[t & 1][0][32 * n + 8 * c + 4 * half]);
                const f32x4 e = BIAS ? *reinterpret_cast<const f32x4 *>(&rows[t & 1][1][32 * n + 8 * c + 4 * half]) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                const f32x4 d = *reinterpret_cast<const f32x4 *>(&rows[t & 1][2][32 * n + 8 * c + 4 * half]);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float x = s[4 * c + r];
                    if constexpr (BIAS) x = __builtin_fmaf(x, a.scale, b[-(8 * c + r)]);
                    x = probability<BIAS>(x, scale, f[r], e[r]);
                    if constexpr (kValuesInLds<T, D>) x = 8 * c + 4 * half + r >= none ? x : 0.0f;
                    s[4 * c + r] = x;
                    dp[4 * c + r] = x * (dp[4 * c + r] - d[r]);
                }
            }
            // (a branch around the masks is the quicker one, but not where registers are short: D of 128, 2709 us without, 3744 with)
            if (!kValuesInLds<T, D> && (mine + 32 > keys || (a.causal && first + offset < mine + 31))) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool in = row_of(r, 0) + 4 * half >= none;
                    s[r] = in ? s[r] : 0.0f;
                    dp[r] = in ? dp[r] : 0.0f;
                }
            }
            sums<T, D>(tile + BYTES, 32 * n, s, dv);
            sums<T, D>(tile, 32 * n, dp, dk);
        }
        if constexpr (BIAS) {
            if (group > 1 && t + 1 < count) {               // the next head's column
                __syncthreads();
                load_column<T>(a, kv * group + (t + 1) % group, column);
                __syncthreads();
            }
        }
        land(t + 1);
    }
    if (j >= a.k_tokens) return;
    if (SPLIT) {
        float *const to = g.dk_parts + (((int64_t)split * a.batch * a.kv_heads + place.unit) * a.k_tokens + j) * 2 * a.head_dim;
        store_row<float, D>(dk, a.scale, to, a.head_dim);
        store_row<float, D>(dv, 1.0f, to + a.head_dim, a.head_dim);
        return;
    }
    store_row<T, D>(dv, 1.0f, static_cast<T *>(g.dv) + batch * g.dv_b + kv * g.dv_h + j * g.dv_t, a.head_dim);
    T *const to = static_cast<T *>(g.dk) + batch * g.dk_b + kv * g.dk_h + j * g.dk_t;
    if (g.dk_d == 1) {
        store_row<T, D>(dk, a.scale, to, a.head_dim);
    } else {                                                // a head's elements apart, its keys beside each other: 32 of them a store
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int d = 32 * n + row_of(r, half);
                if (d >= a.head_dim) continue;
                const float x = dk[n][r] * a.scale;
                if constexpr (sizeof(T) == 4) to[d * g.dk_d] = x;
                else to[d * g.dk_d] = (T)bf16_narrow(x);
            }
    }
}

template <typename T, int D, bool SPLIT>
void launch_queries(const Attention &a, const Gradients &g, int blocks, hipStream_t st)
{
    const unsigned grid = (unsigned)((int64_t)a.batch * a.q_heads * blocks * g.q_splits);
    if (g.parts) launch(queries_kernel<T, D, true, true, SPLIT>, grid, kAttnThreads, 0, st, a, g, blocks);
    else if (a.table) launch(queries_kernel<T, D, true, false, SPLIT>, grid, kAttnThreads, 0, st, a, g, blocks);
    else launch(queries_kernel<T, D, false, false, SPLIT>, grid, kAttnThreads, 0, st, a, g, blocks);
}
template <typename T, int D, bool SPLIT>
void launch_keys(const Attention &a, const Gradients &g, int blocks, hipStream_t st)
{
    const unsigned grid = (unsigned)((int64_t)a.batch * a.kv_heads * blocks * g.k_splits);
    if (a.table) launch(keys_kernel<T, D, true, SPLIT>, grid, kAttnThreads, 0, st, a, g, blocks);
    else launch(keys_kernel<T, D, false, SPLIT>, grid, kAttnThreads, 0, st, a, g, blocks);
}

template <typename T, int D>
void launch_backward(const Attention &a, const Gradients &g, hipStream_t st)
{
    const int k_blocks = (a.k_tokens + kBlock - 1) / kBlock;
    if (a.batch > 0 && g.blocks > 0) {
        if (g.q_splits > 1) launch_queries<T, D, true>(a, g, g.blocks, st);
        else launch_queries<T, D, false>(a, g, g.blocks, st);
    }
    if (a.batch > 0 && k_blocks > 0 && g.all_rows) {
        if (g.k_splits > 1) launch_keys<T, D, true>(a, g, k_blocks, st);
        else launch_keys<T, D, false>(a, g, k_blocks, st);
    }
}

template <typename T>
void attention_backward_of(const Attention &a, const Gradients &g, hipStream_t st)
{
    if (a.head_dim <= 32) launch_backward<T, 32>(a, g, st);
    else if (a.head_dim <= 64) launch_backward<T, 64>(a, g, st);
    else if (a.head_dim <= 96) launch_backward<T, 96>(a, g, st);
    else launch_backward<T, 128>(a, g, st);
}

}  // namespace
}  // namespace slimfit
