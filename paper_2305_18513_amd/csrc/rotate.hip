// Attention's operands out of the rows of a QKV projection, with the norm of each query and key head and the rotation by the
// token's position on the way, the low-bit cache of what their backward pass reads, and that backward pass (not in the
// paper: decoder models' form of the reorderings in heads.hip, keys and values shared by groups of query heads).
//
//   forward   y = rot(x * rstd * gamma), rstd = (mean x^2 + eps)^-1/2; q = q_scale y, k^T = y^T, v = x
//   backward  g = rot^-1(dy), dgamma = sum g x~, dx = rstd (g gamma - x~ mean(g gamma x~)), x~ = x^ rstd
//
// A head's row is L lanes' 16-byte vectors (L a power of two; those past the head's end hold zeros), so that the row's sum
// is a butterfly over L lanes, the element that one is turned with is in the lane's own vector or in that of one lane, and a
// quantisation block is block / E lanes.  A workgroup owns 1024 / L rows (token by token, batch by batch) in four passes,
// whose blocks' divisions a quad of lanes shares, and one head of the keys, or several of the queries or values one after
// the other, with the angles of its rows held in registers for all of them.  Keys go through LDS (rows an odd number of
// words apart) into their transposed place: 16 bytes along the tokens where those are aligned, single elements otherwise.
#include "elements.hpp"

namespace slimfit {
namespace {

constexpr int kThreads = 256;
constexpr int kPasses = 4;
constexpr int kTileWords = 4096 + 256;     // 1024 / L rows of 4 L + 1 words, L >= 4

struct Shape {
    uint32_t rows, tokens, q_heads, kv_heads, dim;         // rows = batch * tokens
    uint32_t per, q_units, units;                          // heads a query (or value) unit, units of queries, of all
    uint32_t positions, half;                              // half = rotary_dim / 2; 0: no rotation
    uint32_t adjacent, norm;
    int group, block_shift;                                // lanes of a quantisation block; log2 of its elements
    float eps, inv_dim, q_scale;
    Divide by_tokens, by_dim, by_units;
};

// cos and signed sin of the E elements at e0 of a row: turned(y)[i] = y[i] c[i] + partner(y)[i] s[i]
template <int E>
__device__ __forceinline__ void load_angles(const float *__restrict__ table, const int32_t *__restrict__ ids, const Shape &z, uint32_t row, uint32_t t,
                                            uint32_t e0, float (&c)[E], float (&s)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
    if (row >= z.rows || e0 >= 2 * z.half) return;
    const uint32_t place = ids ? (uint32_t)ids[row] : t;
    if (place >= z.positions) return;                      // padding
    const float *at = table + (int64_t)place * (2 * z.half);
    if (z.adjacent) {
        at += e0 / 2;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            c[i] = at[i / 2];
            s[i] = i % 2 ? at[z.half + i / 2] : -at[z.half + i / 2];
        }
    } else {
        const bool low = e0 < z.half;
        at += low ? e0 : e0 - z.half;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            c[i] = at[i];
            s[i] = low ? -at[z.half + i] : at[z.half + i];
        }
    }
}
// from: the lane that holds the partners (its own where the pairs are neighbours or nothing is turned).  BACK: by the angle back.
template <int E, bool BACK>
__device__ __forceinline__ void turn(float (&y)[E], const float (&c)[E], const float (&s)[E], int from, const Shape &z)
{
    if (z.half == 0) return;
    float other[E];
    if (z.adjacent) {
#pragma unroll
        for (int i = 0; i < E; ++i) other[i] = y[i ^ 1];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            other[i] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(from * 4, __builtin_bit_cast(int, y[i])));
    }
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = fmaf(other[i], BACK ? -s[i] : s[i], y[i] * c[i]);
}

// A workgroup's rows of one key head between their two layouts.  One thread moves E tokens (of two elements in bf16) where
// every token row begins on 16 bytes, one element otherwise.
template <typename T, int ROWS, bool IN>
__device__ __forceinline__ void through_tile(uint32_t *tile, uint32_t pitch, T *kt, const Shape &z, uint32_t row0, uint32_t head)
{
    constexpr int E = Vec<T>::V, WIDE = sizeof(T) == 2 ? 2 : 1;
    auto place = [&](uint32_t row, uint32_t d) {           // of element d of this head of a token
        const uint32_t b = z.by_tokens(row), t = row - b * z.tokens;
        return kt + (((int64_t)b * z.kv_heads + head) * z.dim + d) * z.tokens + t;
    };
    if (z.tokens % E == 0) {
        constexpr uint32_t CHUNKS = ROWS / E;
        for (uint32_t i = threadIdx.x; i < CHUNKS * (z.dim / WIDE); i += kThreads) {
            const uint32_t r = i % CHUNKS * E, d = i / CHUNKS * WIDE;
            if (row0 + r >= z.rows) continue;              // (rows is a multiple of E)
            T *at = place(row0 + r, d);
            uint32_t *words = tile + r * pitch + d / WIDE;
            if constexpr (WIDE == 1) {
                if constexpr (IN) {
                    const u32x4 v = load_global<true>(reinterpret_cast<const u32x4 *>(at));
#pragma unroll
                    for (int e = 0; e < E; ++e) words[e * pitch] = v[e];
                } else {
                    u32x4 v;
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = words[e * pitch];
                    store_global<true>(reinterpret_cast<u32x4 *>(at), v);
                }
            } else {
                if constexpr (IN) {
                    const u32x4 a = load_global<true>(reinterpret_cast<const u32x4 *>(at));
                    const u32x4 b = load_global<true>(reinterpret_cast<const u32x4 *>(at + z.tokens));
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        words[e * pitch] = __builtin_amdgcn_perm(b[e / 2], a[e / 2], 0x05040100u);
                        words[(e + 1) * pitch] = __builtin_amdgcn_perm(b[e / 2], a[e / 2], 0x07060302u);
                    }
                } else {
                    u32x4 a, b;
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        const uint32_t x = words[e * pitch], y = words[(e + 1) * pitch];
                        a[e / 2] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                        b[e / 2] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                    }
                    store_global<true>(reinterpret_cast<u32x4 *>(at), a);
                    store_global<true>(reinterpret_cast<u32x4 *>(at + z.tokens), b);
                }
            }
        }
        return;
    }
    T *elements = reinterpret_cast<T *>(tile);
    const uint32_t step = pitch * (4 / sizeof(T));
    const bool along = z.tokens >= 8;                      // along the tokens, or (few of them) along the elements
    for (uint32_t i = threadIdx.x; i < ROWS * z.dim; i += kThreads) {
        const uint32_t q = along ? i / ROWS : z.by_dim(i);
        const uint32_t r = along ? i % ROWS : q, d = along ? q : i - q * z.dim;
        if (row0 + r >= z.rows) continue;
        if constexpr (IN) elements[r * step + d] = *place(row0 + r, d);
        else *place(row0 + r, d) = elements[r * step + d];
    }
}

template <typename T, int L, int BITS>
__global__ void __launch_bounds__(kThreads)
forward_kernel(const T *__restrict__ qkv, const float *__restrict__ gamma_q, const float *__restrict__ gamma_k, const float *__restrict__ table,
               const int32_t *__restrict__ ids, T *__restrict__ q, T *__restrict__ kt, T *__restrict__ v, float *__restrict__ rstd,
               uint8_t *__restrict__ codes, float *__restrict__ scales, Shape z, uint32_t first)
{
    using raw = typename Vec<T>::raw;
    constexpr int E = Vec<T>::V, SLOTS = kThreads / L, ROWS = SLOTS * kPasses;
    __shared__ uint32_t tile[kTileWords];
    const uint32_t at = first + blockIdx.x, tiled = z.by_units(at), unit = at - tiled * z.units, row0 = tiled * ROWS;
    const uint32_t lane = threadIdx.x % L, slot = threadIdx.x / L, e0 = lane * E;
    const bool in_head = e0 < z.dim;
    const uint32_t every = z.q_heads + 2 * z.kv_heads, normed = z.q_heads + z.kv_heads;
    uint32_t row[kPasses], batch[kPasses], token[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        row[p] = row0 + p * SLOTS + slot;
        batch[p] = z.by_tokens(row[p]);
        token[p] = row[p] - batch[p] * z.tokens;
    }
    auto load = [&](uint32_t head, raw(&to)[kPasses]) {    // head of the projection's row
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            to[p] = raw{};
            if (row[p] < z.rows && in_head) to[p] = load_global<true>(reinterpret_cast<const raw *>(qkv + ((int64_t)row[p] * every + head) * z.dim + e0));
        }
    };
    if (unit >= z.q_units + z.kv_heads) {                  // values
        const uint32_t h0 = (unit - z.q_units - z.kv_heads) * z.per, h1 = min(h0 + z.per, z.kv_heads);
        for (uint32_t h = h0; h < h1; ++h) {
            raw x[kPasses];
            load(normed + h, x);
#pragma unroll
            for (int p = 0; p < kPasses; ++p)
                if (row[p] < z.rows && in_head)
                    store_global<true>(reinterpret_cast<raw *>(v + (((int64_t)batch[p] * z.kv_heads + h) * z.tokens + token[p]) * z.dim + e0), x[p]);
        }
        return;
    }
    const bool key = unit >= z.q_units;
    const uint32_t h0 = key ? z.q_heads + unit - z.q_units : unit * z.per, h1 = key ? h0 + 1 : min(h0 + z.per, z.q_heads);
    float c[kPasses][E], s[kPasses][E], gamma[E];
    const int mine = threadIdx.x & (kWave - 1);
    int from = mine;
    if (!z.adjacent && e0 < 2 * z.half) from += (e0 < z.half ? 1 : -1) * (int)(z.half / E);
#pragma unroll
    for (int p = 0; p < kPasses; ++p) load_angles<E>(table, ids, z, row[p], token[p], e0, c[p], s[p]);
    const float factor = key ? 1.0f : z.q_scale;
    {
        const float *g = key ? gamma_k : gamma_q;
#pragma unroll
        for (int i = 0; i < E; ++i) gamma[i] = z.norm && in_head ? g[e0 + i] : 1.0f;
    }
    const uint32_t pitch = z.dim * sizeof(T) / 4 + 1;
    for (uint32_t h = h0; h < h1; ++h) {
        raw x[kPasses];
        load(h, x);
        float f[kPasses][E];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) Vec<T>::unpack(x[p], f[p]);
        if constexpr (BITS != 0) {
            uint32_t a[kPasses];
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                float m = 0.0f;
#pragma unroll
                for (int i = 0; i < E; ++i) m = fmaxf(m, fabsf(f[p][i]));
                a[p] = group_max_u32(__builtin_bit_cast(uint32_t, m), z.group);
            }
            float mult[kPasses], scale;
            quad_scales<BITS, kPasses>(a, (int)threadIdx.x, mult, scale);
            const uint32_t own = threadIdx.x & (z.group - 1), own_row = row0 + own * SLOTS + slot;
            if (own < kPasses && own_row < z.rows && in_head)            // lanes 0 .. 3 of a block store a pass's scale each
                scales[(((int64_t)own_row * normed + h) * z.dim + e0) >> z.block_shift] = scale;
#pragma unroll
            for (int p = 0; p < kPasses; ++p) {
                if (row[p] >= z.rows || !in_head) continue;
                uint32_t w[2];
                pack_codes<BITS, E>(f[p], mult[p], w);
                uint8_t *dst = codes + (((int64_t)row[p] * normed + h) * z.dim + e0) * BITS / 8;
                if (E * BITS == 16) store_global<true>(reinterpret_cast<uint16_t *>(dst), (uint16_t)w[0]);
                else if (E * BITS == 32) store_global<true>(reinterpret_cast<uint32_t *>(dst), w[0]);
                else store_global<true>(reinterpret_cast<u32x2 *>(dst), u32x2{w[0], w[1]});
            }
        }
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (z.norm) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < E; ++i) sum = fmaf(f[p][i], f[p][i], sum);
                const float r = __builtin_amdgcn_rsqf(fmaf(group_sum_f32(sum, L), z.inv_dim, z.eps));
                if (lane == 0 && row[p] < z.rows) rstd[(int64_t)row[p] * normed + h] = r;
#pragma unroll
                for (int i = 0; i < E; ++i) f[p][i] = f[p][i] * r * gamma[i];
            }
            turn<E, false>(f[p], c[p], s[p], from, z);
#pragma unroll
            for (int i = 0; i < E; ++i) f[p][i] *= factor;
            const raw out = Vec<T>::pack(f[p]);
            if (!key) {
                if (row[p] < z.rows && in_head)
                    store_global<true>(reinterpret_cast<raw *>(q + (((int64_t)batch[p] * z.q_heads + h) * z.tokens + token[p]) * z.dim + e0), out);
            } else if (in_head) {
                uint32_t *words = tile + (p * SLOTS + slot) * pitch + lane * 4;
                const u32x4 held = __builtin_bit_cast(u32x4, out);
#pragma unroll
                for (int i = 0; i < 4; ++i) words[i] = held[i];
            }
        }
    }
    if (key) {                                             // (uniform for the workgroup)
        __syncthreads();
        through_tile<T, ROWS, false>(tile, pitch, kt, z, row0, h0 - z.q_heads);
    }
}

// partial: [units of queries, units of keys] x row tiles x dim sums of a workgroup each, or null where they are not asked for
template <typename T, int L, int BITS>
__global__ void __launch_bounds__(kThreads)
backward_kernel(const T *__restrict__ dq, const T *__restrict__ dkt, const T *__restrict__ dv, const T *__restrict__ qkv, const uint8_t *__restrict__ codes,
                const float *__restrict__ scales, const float *__restrict__ rstd, const float *__restrict__ gamma_q, const float *__restrict__ gamma_k,
                const float *__restrict__ table, const int32_t *__restrict__ ids, T *__restrict__ dqkv, float *__restrict__ partial, Shape z, uint32_t first)
{
    using raw = typename Vec<T>::raw;
    constexpr int E = Vec<T>::V, SLOTS = kThreads / L, ROWS = SLOTS * kPasses;
    __shared__ uint32_t tile[kTileWords];
    const uint32_t at = first + blockIdx.x, tiled = z.by_units(at), unit = at - tiled * z.units, row0 = tiled * ROWS;
    const uint32_t lane = threadIdx.x % L, slot = threadIdx.x / L, e0 = lane * E;
    const bool in_head = e0 < z.dim;
    const uint32_t every = z.q_heads + 2 * z.kv_heads, normed = z.q_heads + z.kv_heads;
    uint32_t row[kPasses], batch[kPasses], token[kPasses];
    bool has[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        row[p] = row0 + p * SLOTS + slot;
        batch[p] = z.by_tokens(row[p]);
        token[p] = row[p] - batch[p] * z.tokens;
        has[p] = row[p] < z.rows && in_head;
    }
    if (unit >= z.q_units + z.kv_heads) {                  // values
        const uint32_t h0 = (unit - z.q_units - z.kv_heads) * z.per, h1 = min(h0 + z.per, z.kv_heads);
        for (uint32_t h = h0; h < h1; ++h) {
            raw x[kPasses];
#pragma unroll
            for (int p = 0; p < kPasses; ++p)
                if (has[p]) x[p] = load_global<true>(reinterpret_cast<const raw *>(dv + (((int64_t)batch[p] * z.kv_heads + h) * z.tokens + token[p]) * z.dim + e0));
#pragma unroll
            for (int p = 0; p < kPasses; ++p)
                if (has[p]) store_global<true>(reinterpret_cast<raw *>(dqkv + ((int64_t)row[p] * every + normed + h) * z.dim + e0), x[p]);
        }
        return;
    }
    const bool key = unit >= z.q_units;
    const uint32_t h0 = key ? z.q_heads + unit - z.q_units : unit * z.per, h1 = key ? h0 + 1 : min(h0 + z.per, z.q_heads);
    const uint32_t pitch = z.dim * sizeof(T) / 4 + 1;
    if (key) through_tile<T, ROWS, true>(tile, pitch, const_cast<T *>(dkt), z, row0, h0 - z.q_heads);
    float c[kPasses][E], s[kPasses][E], gamma[E], sum_gamma[E];
    const int mine = threadIdx.x & (kWave - 1);
    int from = mine;
    if (!z.adjacent && e0 < 2 * z.half) from += (e0 < z.half ? 1 : -1) * (int)(z.half / E);
#pragma unroll
    for (int p = 0; p < kPasses; ++p) load_angles<E>(table, ids, z, row[p], token[p], e0, c[p], s[p]);
    const float factor = key ? 1.0f : z.q_scale;
    {
        const float *g = key ? gamma_k : gamma_q;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            gamma[i] = z.norm && in_head ? g[e0 + i] : 1.0f;
            sum_gamma[i] = 0.0f;
        }
    }
    if (key) __syncthreads();
    for (uint32_t h = h0; h < h1; ++h) {
        raw grad[kPasses], x[kPasses];
        uint32_t w[kPasses][2];
        float step[kPasses], r[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            grad[p] = x[p] = raw{};
            w[p][0] = w[p][1] = 0u;
            step[p] = r[p] = 0.0f;
            if (!has[p]) continue;
            if (key) {
                const uint32_t *words = tile + (p * SLOTS + slot) * pitch + lane * 4;
                grad[p] = __builtin_bit_cast(raw, u32x4{words[0], words[1], words[2], words[3]});
            } else {
                grad[p] = load_global<true>(reinterpret_cast<const raw *>(dq + (((int64_t)batch[p] * z.q_heads + h) * z.tokens + token[p]) * z.dim + e0));
            }
            if (!z.norm) continue;
            const int64_t element = ((int64_t)row[p] * normed + h) * z.dim + e0;
            if constexpr (BITS == 0) {
                x[p] = load_global<true>(reinterpret_cast<const raw *>(qkv + ((int64_t)row[p] * every + h) * z.dim + e0));
            } else {
                const uint8_t *src = codes + element * BITS / 8;
                if (E * BITS == 16) w[p][0] = load_global<true>(reinterpret_cast<const uint16_t *>(src));
                else if (E * BITS == 32) w[p][0] = load_global<true>(reinterpret_cast<const uint32_t *>(src));
                else { const u32x2 t = load_global<true>(reinterpret_cast<const u32x2 *>(src)); w[p][0] = t.x; w[p][1] = t.y; }
                step[p] = scales[element >> z.block_shift];
            }
            r[p] = rstd[(int64_t)row[p] * normed + h];
        }
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            float g[E];
            Vec<T>::unpack(grad[p], g);
#pragma unroll
            for (int i = 0; i < E; ++i) g[i] *= factor;
            turn<E, true>(g, c[p], s[p], from, z);
            if (z.norm) {
                float xn[E], dot = 0.0f;
                if constexpr (BITS == 0) {
                    Vec<T>::unpack(x[p], xn);
                } else {
#pragma unroll
                    for (int i = 0; i < E; ++i) xn[i] = (float)code_field<BITS>(w[p][i * BITS / 32], i % (32 / BITS)) * step[p];
                }
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    xn[i] *= r[p];
                    sum_gamma[i] = fmaf(g[i], xn[i], sum_gamma[i]);
                    g[i] *= gamma[i];
                    dot = fmaf(g[i], xn[i], dot);
                }
                dot = group_sum_f32(dot, L) * z.inv_dim;
#pragma unroll
                for (int i = 0; i < E; ++i) g[i] = r[p] * fmaf(-xn[i], dot, g[i]);
            }
            if (has[p]) store_global<true>(reinterpret_cast<raw *>(dqkv + ((int64_t)row[p] * every + h) * z.dim + e0), Vec<T>::pack(g));
        }
    }
    if (partial) {                                         // (uniform for the launch)
        __syncthreads();                                   // the tile is read
        float *sums = reinterpret_cast<float *>(tile);     // SLOTS x dim
        if (in_head) {
#pragma unroll
            for (int i = 0; i < E; ++i) sums[slot * z.dim + e0 + i] = sum_gamma[i];
        }
        __syncthreads();
        const uint32_t tiles = (z.rows + ROWS - 1) / ROWS;
        float *to = partial + ((int64_t)unit * tiles + tiled) * z.dim;
        for (uint32_t d = threadIdx.x; d < z.dim; d += kThreads) {
            float total = 0.0f;
            for (int k = 0; k < SLOTS; ++k) total += sums[k * z.dim + d];
            to[d] = total;
        }
    }
}

// dgamma[d] = sum over the partial sums of its side.  A workgroup: 16 columns, 16 slices of the rows.
__global__ void __launch_bounds__(kThreads)
gamma_kernel(const float *__restrict__ partial, uint32_t dim, int64_t q_rows, int64_t k_rows, float *__restrict__ dgamma_q, float *__restrict__ dgamma_k)
{
    __shared__ double sums[kThreads];
    const uint32_t blocks = gridDim.x / 2, side = blockIdx.x / blocks, d = blockIdx.x % blocks * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
    const float *from = partial + (side ? q_rows * dim : 0);
    const int64_t n = side ? k_rows : q_rows;
    double total = 0.0;
    if (d < dim) {
#pragma unroll 8
        for (int64_t i = slice; i < n; i += 16) total += (double)from[i * dim + d];
    }
    sums[threadIdx.x] = total;
    __syncthreads();
    if (slice == 0 && d < dim) {
        for (int k = 1; k < 16; ++k) total += sums[k * 16 + threadIdx.x];
        (side ? dgamma_k : dgamma_q)[d] = (float)total;
    }
}

int lanes_of(int32_t dt, int32_t dim)
{
    const int vectors = dim / (dt == SLIMFIT_F32 ? 4 : 8);
    int L = 4;
    while (L < vectors) L *= 2;
    return L;
}

// Heads a query (or value) workgroup takes one after the other: as many as leave four workgroups to a compute unit, at most 8.
int heads_each(int64_t tiles, int32_t heads)
{
    int per = 8;
    while (per > 1 && tiles * ((heads + per - 1) / per) < 1024) per /= 2;
    return per;
}

int32_t validate(int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim)
{
    if (!dtype_ok(dt) || batch < 0 || tokens < 0 || q_heads < 1 || kv_heads < 1 || dim < 1 || q_heads % kv_heads != 0) return SLIMFIT_ERR_INVALID_ARG;
    if (dim % (dt == SLIMFIT_F32 ? 4 : 8) != 0 || dim > 256) return SLIMFIT_ERR_UNSUPPORTED;
    if (batch == 0 || tokens == 0) return SLIMFIT_OK;
    if (batch >= ((int64_t)1 << 31) / tokens || q_heads > (1 << 20)) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

struct Plan {
    int L, per;
    int64_t tiles, q_units, v_units, blocks;
    Plan(int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim)
    {
        L = lanes_of(dt, dim);
        const int64_t each = 1024 / L;
        tiles = (batch * tokens + each - 1) / each;
        per = heads_each(tiles, q_heads);
        q_units = (q_heads + per - 1) / per;
        v_units = (kv_heads + per - 1) / per;
        blocks = tiles * (q_units + kv_heads + v_units);
    }
    size_t workspace(int32_t kv_heads, int32_t dim) const { return (size_t)tiles * (size_t)(q_units + kv_heads) * (size_t)dim * 4; }
};

struct Rotation {
    const float *table;
    int32_t positions, rotary_dim, pairing;
    const int32_t *ids;
};

int32_t validate_rotation(const Rotation &r, int32_t dt, int64_t batch, int32_t tokens, int32_t dim)
{
    if (r.positions < 0 || r.rotary_dim < 0 || r.rotary_dim > dim) return SLIMFIT_ERR_INVALID_ARG;
    if (r.rotary_dim == 0) return SLIMFIT_OK;
    if (r.pairing != SLIMFIT_ROTARY_HALVES && r.pairing != SLIMFIT_ROTARY_ADJACENT) return SLIMFIT_ERR_INVALID_ARG;
    if (r.rotary_dim % (dt == SLIMFIT_F32 ? 8 : 16) != 0) return SLIMFIT_ERR_UNSUPPORTED;
    if (batch == 0 || tokens == 0) return SLIMFIT_OK;
    if ((!r.table && r.positions > 0) || (!r.ids && r.positions < tokens)) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(r.table, 16) || !aligned_to(r.ids, 4)) return SLIMFIT_ERR_ALIGNMENT;
    return SLIMFIT_OK;
}
int32_t validate_cache(int32_t bits, int32_t block, int32_t dim, bool norm)
{
    if (bits == 0) return SLIMFIT_OK;
    if (!norm) return SLIMFIT_ERR_INVALID_ARG;
    if ((bits != 4 && bits != 8) || (block != 32 && block != 64 && block != 128 && block != 256) || dim % block != 0) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}
int32_t check_rotation(const Rotation &r, int64_t rows)
{
    if (r.rotary_dim == 0) return SLIMFIT_OK;
    int32_t rc = check_device_range(r.table, (size_t)r.positions * (size_t)r.rotary_dim * 4);
    if (rc == SLIMFIT_OK && r.ids) rc = check_device_range(r.ids, (size_t)rows * 4);
    return rc;
}

Shape shape_of(const Plan &p, const Rotation &r, int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim, bool norm,
               float eps, float q_scale, int32_t bits, int32_t block)
{
    const uint32_t units = (uint32_t)(p.q_units + kv_heads + p.v_units);
    Shape z = {(uint32_t)(batch * tokens), (uint32_t)tokens, (uint32_t)q_heads, (uint32_t)kv_heads, (uint32_t)dim, (uint32_t)p.per, (uint32_t)p.q_units,
               units, (uint32_t)r.positions, (uint32_t)r.rotary_dim / 2, r.pairing == SLIMFIT_ROTARY_ADJACENT, norm, 4, 0, eps, 1.0f / (float)dim, q_scale,
               Divide((uint32_t)tokens), Divide((uint32_t)dim), Divide(units)};
    if (bits != 0) {
        z.group = block / (dt == SLIMFIT_F32 ? 4 : 8);
        z.block_shift = __builtin_ctz((unsigned)block);
    }
    return z;
}

// f(T{}, L, BITS) for the call's type, lanes a head and bits
template <typename F>
void choose(int32_t dt, int L, int32_t bits, F f)
{
    auto with_bits = [&](auto t, auto l) {
        if (bits == 0) f(t, l, std::integral_constant<int, 0>{});
        else if (bits == 4) f(t, l, std::integral_constant<int, 4>{});
        else f(t, l, std::integral_constant<int, 8>{});
    };
    auto with_lanes = [&](auto t) {
        switch (L) {
        case 4: with_bits(t, std::integral_constant<int, 4>{}); break;
        case 8: with_bits(t, std::integral_constant<int, 8>{}); break;
        case 16: with_bits(t, std::integral_constant<int, 16>{}); break;
        default:
            if constexpr (sizeof(t) == 4) {
                if (L == 64) { with_bits(t, std::integral_constant<int, 64>{}); break; }
            }
            with_bits(t, std::integral_constant<int, 32>{});
        }
    };
    if (dt == SLIMFIT_F32) with_lanes(float{});
    else with_lanes(uint16_t{});
}

}  // namespace
}  // namespace slimfit

using namespace slimfit;

extern "C" int32_t slimfit_heads_norm_rotate_forward(const void *qkv, int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads,
                                                     int32_t head_dim, const float *gamma_q, const float *gamma_k, float eps, const float *table,
                                                     int32_t positions, int32_t rotary_dim, int32_t pairing, const int32_t *position_ids,
                                                     float q_scale, int32_t bits, int32_t block, void *q, void *kt, void *v, float *rstd,
                                                     uint8_t *codes, float *scales, void *stream)
{
    StreamScope capture_aware(stream);
    const Rotation turn = {table, positions, rotary_dim, pairing, position_ids};
    const bool norm = gamma_q != nullptr;
    int32_t rc = validate(dt, batch, tokens, q_heads, kv_heads, head_dim);
    if (rc != SLIMFIT_OK) return rc;
    if ((gamma_q == nullptr) != (gamma_k == nullptr) || (norm && !(eps >= 0.0f))) return SLIMFIT_ERR_INVALID_ARG;
    if ((rc = validate_rotation(turn, dt, batch, tokens, head_dim)) != SLIMFIT_OK) return rc;
    if ((rc = validate_cache(bits, block, head_dim, norm)) != SLIMFIT_OK) return rc;
    if (batch == 0 || tokens == 0) return SLIMFIT_OK;
    if (!qkv || !q || !kt || !v || (norm && !rstd) || (bits != 0 && (!codes || !scales))) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(qkv, 16) || !aligned_to(q, 16) || !aligned_to(kt, 16) || !aligned_to(v, 16) ||
        (norm && (!aligned_to(gamma_q, 16) || !aligned_to(gamma_k, 16) || !aligned_to(rstd, 4))) ||
        (bits != 0 && (!aligned_to(codes, 16) || !aligned_to(scales, 16))))
        return SLIMFIT_ERR_ALIGNMENT;
    const Plan plan(dt, batch, tokens, q_heads, kv_heads, head_dim);
    if (plan.blocks > 0x7FFFFFFFLL) return SLIMFIT_ERR_UNSUPPORTED;
    const size_t rows = (size_t)(batch * tokens), head = (size_t)head_dim * dtype_size(dt), normed = (size_t)q_heads + (size_t)kv_heads;
    const size_t in = rows * (normed + (size_t)kv_heads) * head, q_bytes = rows * (size_t)q_heads * head, k_bytes = rows * (size_t)kv_heads * head;
    if (meet(qkv, in, q, q_bytes) || meet(qkv, in, kt, k_bytes) || meet(qkv, in, v, k_bytes) || meet(q, q_bytes, kt, k_bytes) ||
        meet(q, q_bytes, v, k_bytes) || meet(kt, k_bytes, v, k_bytes))
        return SLIMFIT_ERR_INVALID_ARG;
    if ((rc = check_device_range(qkv, in)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(q, q_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(kt, k_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(v, k_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_rotation(turn, (int64_t)rows)) != SLIMFIT_OK) return rc;
    if (norm) {
        if ((rc = check_device_range(gamma_q, (size_t)head_dim * 4)) != SLIMFIT_OK) return rc;
        if ((rc = check_device_range(gamma_k, (size_t)head_dim * 4)) != SLIMFIT_OK) return rc;
        if ((rc = check_device_range(rstd, rows * normed * 4)) != SLIMFIT_OK) return rc;
    }
    if (bits != 0) {
        const size_t n = rows * normed * (size_t)head_dim;
        if ((rc = check_device_range(codes, n * (size_t)bits / 8)) != SLIMFIT_OK) return rc;
        if ((rc = check_device_range(scales, n / (size_t)block * 4)) != SLIMFIT_OK) return rc;
    }
    const Shape z = shape_of(plan, turn, dt, batch, tokens, q_heads, kv_heads, head_dim, norm, eps, q_scale, bits, block);
    hipStream_t st = static_cast<hipStream_t>(stream);
    constexpr int64_t kMost = kMaxGridThreads / kThreads;
    for (int64_t first = 0; first < plan.blocks; first += kMost) {
        const unsigned here = (unsigned)(plan.blocks - first < kMost ? plan.blocks - first : kMost);
        choose(dt, plan.L, bits, [&](auto t, auto l, auto b) {
            using T = decltype(t);
            launch(forward_kernel<T, decltype(l)::value, decltype(b)::value>, here, kThreads, 0, st, static_cast<const T *>(qkv), gamma_q, gamma_k, table,
                   position_ids, static_cast<T *>(q), static_cast<T *>(kt), static_cast<T *>(v), rstd, codes, scales, z, (uint32_t)first);
        });
    }
    return launch_status();
}

extern "C" int32_t slimfit_heads_norm_rotate_workspace(int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                                       size_t *bytes)
{
    const int32_t rc = validate(dt, batch, tokens, q_heads, kv_heads, head_dim);
    if (rc != SLIMFIT_OK) return rc;
    if (!bytes) return SLIMFIT_ERR_INVALID_ARG;
    *bytes = batch == 0 || tokens == 0 ? 0 : Plan(dt, batch, tokens, q_heads, kv_heads, head_dim).workspace(kv_heads, head_dim);
    return SLIMFIT_OK;
}

extern "C" int32_t slimfit_heads_norm_rotate_backward(const void *dq, const void *dkt, const void *dv, const void *qkv, const uint8_t *codes,
                                                      const float *scales, int32_t bits, int32_t block, const float *rstd, int32_t dt, int64_t batch,
                                                      int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim, const float *gamma_q,
                                                      const float *gamma_k, const float *table, int32_t positions, int32_t rotary_dim,
                                                      int32_t pairing, const int32_t *position_ids, float q_scale, void *dqkv, float *dgamma_q,
                                                      float *dgamma_k, void *workspace, size_t workspace_bytes, void *stream)
{
    StreamScope capture_aware(stream);
    const Rotation turn = {table, positions, rotary_dim, pairing, position_ids};
    const bool norm = gamma_q != nullptr, want = dgamma_q != nullptr, reads = norm && bits == 0;
    int32_t rc = validate(dt, batch, tokens, q_heads, kv_heads, head_dim);
    if (rc != SLIMFIT_OK) return rc;
    if ((gamma_q == nullptr) != (gamma_k == nullptr) || (dgamma_q == nullptr) != (dgamma_k == nullptr) || (want && !norm)) return SLIMFIT_ERR_INVALID_ARG;
    if ((rc = validate_rotation(turn, dt, batch, tokens, head_dim)) != SLIMFIT_OK) return rc;
    if ((rc = validate_cache(bits, block, head_dim, norm)) != SLIMFIT_OK) return rc;
    if (want && (!aligned_to(dgamma_q, 16) || !aligned_to(dgamma_k, 16))) return SLIMFIT_ERR_ALIGNMENT;
    const bool empty = batch == 0 || tokens == 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto check_gammas = [&]() {
        const int32_t first = check_device_range(dgamma_q, want ? (size_t)head_dim * 4 : 0);
        return first != SLIMFIT_OK ? first : check_device_range(dgamma_k, want ? (size_t)head_dim * 4 : 0);
    };
    const unsigned gamma_blocks = 2u * (unsigned)((head_dim + 15) / 16);
    if (empty) {
        if (!want) return SLIMFIT_OK;
        if ((rc = check_gammas()) != SLIMFIT_OK) return rc;
        launch(gamma_kernel, gamma_blocks, kThreads, 0, st, nullptr, (uint32_t)head_dim, 0, 0, dgamma_q, dgamma_k);      // sums of nothing
        return launch_status();
    }
    if (!dq || !dkt || !dv || !dqkv || (reads && !qkv) || (norm && !rstd) || (bits != 0 && (!codes || !scales))) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(dq, 16) || !aligned_to(dkt, 16) || !aligned_to(dv, 16) || !aligned_to(dqkv, 16) || (reads && !aligned_to(qkv, 16)) ||
        (norm && (!aligned_to(gamma_q, 16) || !aligned_to(gamma_k, 16) || !aligned_to(rstd, 4))) ||
        (bits != 0 && (!aligned_to(codes, 16) || !aligned_to(scales, 16))))
        return SLIMFIT_ERR_ALIGNMENT;
    const Plan plan(dt, batch, tokens, q_heads, kv_heads, head_dim);
    if (plan.blocks > 0x7FFFFFFFLL) return SLIMFIT_ERR_UNSUPPORTED;
    if (want) {
        if (!workspace || workspace_bytes < plan.workspace(kv_heads, head_dim)) return SLIMFIT_ERR_WORKSPACE;
        if (!aligned_to(workspace, 16)) return SLIMFIT_ERR_ALIGNMENT;
    }
    const size_t rows = (size_t)(batch * tokens), head = (size_t)head_dim * dtype_size(dt), normed = (size_t)q_heads + (size_t)kv_heads;
    const size_t out = rows * (normed + (size_t)kv_heads) * head, q_bytes = rows * (size_t)q_heads * head, k_bytes = rows * (size_t)kv_heads * head;
    if (meet(dqkv, out, dq, q_bytes) || meet(dqkv, out, dkt, k_bytes) || meet(dqkv, out, dv, k_bytes) || (reads && meet(dqkv, out, qkv, out)))
        return SLIMFIT_ERR_INVALID_ARG;
    if ((rc = check_gammas()) != SLIMFIT_OK) return rc;
    if (want && (rc = check_device_range(workspace, plan.workspace(kv_heads, head_dim))) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(dqkv, out)) != SLIMFIT_OK) return rc;
    if (reads && (rc = check_device_range(qkv, out)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(dq, q_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(dkt, k_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(dv, k_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_rotation(turn, (int64_t)rows)) != SLIMFIT_OK) return rc;
    if (norm) {
        if ((rc = check_device_range(gamma_q, (size_t)head_dim * 4)) != SLIMFIT_OK) return rc;
        if ((rc = check_device_range(gamma_k, (size_t)head_dim * 4)) != SLIMFIT_OK) return rc;
        if ((rc = check_device_range(rstd, rows * normed * 4)) != SLIMFIT_OK) return rc;
    }
    if (bits != 0) {
        const size_t n = rows * normed * (size_t)head_dim;
        if ((rc = check_device_range(codes, n * (size_t)bits / 8)) != SLIMFIT_OK) return rc;
        if ((rc = check_device_range(scales, n / (size_t)block * 4)) != SLIMFIT_OK) return rc;
    }
    const Shape z = shape_of(plan, turn, dt, batch, tokens, q_heads, kv_heads, head_dim, norm, 0.0f, q_scale, bits, block);
    float *partial = want ? static_cast<float *>(workspace) : nullptr;
    constexpr int64_t kMost = kMaxGridThreads / kThreads;
    for (int64_t first = 0; first < plan.blocks; first += kMost) {
        const unsigned here = (unsigned)(plan.blocks - first < kMost ? plan.blocks - first : kMost);
        choose(dt, plan.L, bits, [&](auto t, auto l, auto b) {
            using T = decltype(t);
            launch(backward_kernel<T, decltype(l)::value, decltype(b)::value>, here, kThreads, 0, st, static_cast<const T *>(dq),
                   static_cast<const T *>(dkt), static_cast<const T *>(dv), static_cast<const T *>(qkv), codes, scales, rstd, gamma_q, gamma_k, table,
                   position_ids, static_cast<T *>(dqkv), partial, z, (uint32_t)first);
        });
    }
    if (want)
        launch(gamma_kernel, gamma_blocks, kThreads, 0, st, partial, (uint32_t)head_dim, plan.tiles * plan.q_units, plan.tiles * (int64_t)kv_heads, dgamma_q,
               dgamma_k);
    return launch_status();
}
