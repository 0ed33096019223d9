// What the attention kernels share (attention_forward.hip, attention_backward.hip).
//
// A wave holds 32 rows of its own in registers (queries in the forward pass and for dq, keys for dk and dv) and goes over tiles of the
// other side's rows, which the workgroup lays into LDS as they lie in memory.  Two products carry everything:
//   dots   s[t][o] = sum over d of tile[t][d] own[o][d]:  the tile's rows are the matrix instructions' first operand, 16 bytes of a row a
//          lane, the wave's own rows the second, already in that form.  Lane l gets column o = l % 32 and the rows
//          t = 8 (r / 4) + 4 (l / 32) + r % 4 of 32, r = 0 .. 15 (`row_of`).
//   sums   out[d][o] += sum over t of tile[t][d] x[t][o]:  x is a function of s, which lies as the second operand wants it (the order of
//          the sum is free, so lanes keep their rows); the first is the tile read across (ds_read_b64_tr_b16; fp32: one element
//          a lane).  Nothing goes through LDS or other lanes on the way from s to out.
// bf16: v_mfma_f32_32x32x16_bf16, fp32: v_mfma_f32_32x32x2_f32.  Rows past the end, and elements past a head's, are zeros by the bounds
// of the buffer descriptors.
#pragma once

#include "common.hpp"

namespace slimfit {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = 4;
constexpr int kOwn = 32;                     // rows of a wave
constexpr int kBlock = kOwn * kAttnWaves;    // rows of a workgroup
constexpr int kTile = 64;                    // rows of a tile
constexpr int kFewTile = 128;                // keys of a tile of the kernel for few queries, 32 a wave
constexpr int kMostSplits = 64;              // workgroups that share a sequence's keys out there
constexpr int kDistances = kBlock + kTile;   // distances between a workgroup's rows and a tile's, and one
constexpr int kMostBuckets = 1024;
constexpr int kMostHeadDim = 128;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// One operand: element (batch, head, token, d) is at[batch * b + head * h + token * t + d].
struct Operand {
    const void *at;
    int64_t b, h, t;
};

struct Attention {
    Operand q, k, v;
    int32_t batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, causal, buckets;
    float scale;
    const int32_t *lengths;                  // [batch] or NULL
    const void *table;                       // [buckets, q_heads] of the operands' type, or NULL
    const int32_t *bucket_of;                // [q_tokens + k_tokens - 1]
};

// keys of a sequence
__device__ __forceinline__ int keys_of(const Attention &a, int batch)
{
    return a.lengths ? min(max(a.lengths[batch], 0), a.k_tokens) : a.k_tokens;
}
// keys that query i sees, of `keys`: those before
__device__ __forceinline__ int seen_by(const Attention &a, int i, int keys)
{
    return a.causal ? min(keys, max(0, i + 1 + a.k_tokens - a.q_tokens)) : keys;
}
// the first of `all` tiles that the `split`-th of `splits` goes over; the next one's is its end
__host__ __device__ __forceinline__ int first_of(int all, int split, int splits) { return (int)((int64_t)all * split / splits); }
// tiles of keys that the 128 queries from q0 on see
__device__ __forceinline__ int key_tiles(const Attention &a, int q0, int keys)
{
    return (seen_by(a, min(q0 + kBlock, a.q_tokens) - 1, keys) + kTile - 1) / kTile;
}

// Workgroups go to the eight XCDs in turn, and each has its own L2: the work of one pair of sequence and key head, whose `each` times
// `blocks` workgroups read the same keys and values (or queries), stays on one.  There the pairs go one after another or, where blocks
// differ in length (causal), the first block of all of them, then the second, so that what is left at the end is short.  (2048 x 2048 by
// 128 causal, 32 heads on 8, 8 sequences: 370 us in the grid's order, 317 to 335 so; 1024 x 1024 by 64 causal 61, 60.)
struct Place {
    int unit, block, in;
    __device__ __forceinline__ Place(int units, int blocks, int each, bool by_block)
    {
        const int b = (int)blockIdx.x, whole = units / 8, first = whole * 8 * blocks * each;
        int n = b / 8, xcd = b % 8, here = whole, step = 8, base = 0;
        if (b >= first) {                                   // the last few pairs go round all XCDs
            n = b - first;
            xcd = 0;
            here = units % 8;
            step = 1;
            base = whole * 8;
        }
        in = n % each;
        n /= each;
        const int local = by_block ? n % here : n / blocks;
        block = by_block ? n / here : n % blocks;
        unit = base + xcd + local * step;
    }
};

typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_at(const void *at, int64_t bytes)        // reads past its end give 0
{
    const int64_t most = 0xFFFFFFF0LL, n = bytes < 0 ? 0 : bytes < most ? bytes : most;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, (int)(uint32_t)n, 0x00020000);
}
__device__ __forceinline__ u32x4 load16(Buffer b, int at)
{
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0);
    return u32x4{v[0], v[1], v[2], v[3]};
}
constexpr int kNowhere = -16;                // an offset past every descriptor's end

template <typename T> constexpr int kPerVector = 16 / (int)sizeof(T);
// A tile's rows in LDS.  fp32: 16 bytes more than a row holds, so that rows' vectors begin four banks apart.  bf16: rows of 4, 8 or 16
// vectors whose places are exchanged by the row (`turn_of`): sixteen rows' vectors of the same number, which `dots` reads at a
// time, lie in different banks, and so do four rows' of four beside each other, which `across` reads (with the padding instead
// half of the reads' time went into conflicts, 52 of 104 million cycles of 2048 x 2048 by 128 and 256 heads).
template <typename T, int D> constexpr int kRowVectors = D / kPerVector<T> == 12 ? 16 : D / kPerVector<T>;
template <typename T, int D> constexpr int kPitch = sizeof(T) == 4 ? D * 4 + 16 : kRowVectors<T, D> * 16;
template <typename T, int D> constexpr int kTileBytes = kTile * kPitch<T, D>;
template <typename T, int D>
__device__ __forceinline__ int turn_of(int row)
{
    if constexpr (sizeof(T) == 4) return 0;
    else if constexpr (kRowVectors<T, D> == 16) return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (kRowVectors<T, D> == 8) return ((row & 2) << 1) | ((row >> 2) & 3);
    else return (row >> 2) & 3;
}

// rows [first, first + count) of a head, `row` elements apart, from its first element on
template <typename T>
__device__ __forceinline__ Buffer rows_from(const T *head, int64_t row, int first, int count, int dim)
{
    return buffer_at(head + first * row, count > 0 ? ((count - 1) * row + dim) * (int64_t)sizeof(T) : 0);
}

// One side's tiles on their way from memory to LDS: `fetch` asks for the tile where this stands, `land` (and, after all of them, `landed`)
// makes it whole; what lies in its place has to be through before the fetch.  bf16 goes straight to LDS, each lane's 16 bytes to the
// next place of the wave's kilobyte, asked for from where they belong; fp32, whose rows are padded, through registers.  A step
// from tile to tile is two additions (with addresses formed anew for each tile scalar instructions were a fourth of the loops).
template <typename T, int D, int ROWS = kTile>
struct Tiles {
    static constexpr bool DIRECT = sizeof(T) == 2;
    static constexpr int VECTORS = DIRECT ? kRowVectors<T, D> : D / kPerVector<T>, EACH = ROWS * VECTORS / kAttnThreads;
    static_assert(ROWS * VECTORS % kAttnThreads == 0, "every thread takes as many");
    int from[EACH];
    u32x4 held[DIRECT ? 1 : EACH];
    uint64_t at;                             // the tile's first element
    int64_t left, step;                      // bytes from there to the end of what there is; from a tile to the next

    __device__ __forceinline__ static int vector(int i)     // the thread's i-th of the tile's vectors
    {
        return DIRECT ? ((int)(threadIdx.x >> 6) * EACH + i) * kWave + (int)(threadIdx.x & 63) : (int)threadIdx.x + i * kAttnThreads;
    }
    // rows [0, end) of a head, `row` elements apart, from row `first` on
    __device__ __forceinline__ void start(const T *head, int64_t row, int first, int end, int dim)
    {
        at = reinterpret_cast<uint64_t>(head + first * row);
        left = end > 0 ? ((end - 1 - first) * row + dim) * (int64_t)sizeof(T) : 0;
        step = ROWS * row * (int64_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int r = vector(i) / VECTORS, c = (vector(i) % VECTORS) ^ turn_of<T, D>(r);
            from[i] = c * kPerVector<T> < dim ? r * ((int)row * (int)sizeof(T)) + c * 16 : kNowhere;
        }
    }
    __device__ __forceinline__ void forward() { at += step; left -= step; }
    __device__ __forceinline__ void fetch(char *lds)
    {
        const int64_t bytes = left < 0 ? 0 : left < 0xFFFFFFF0LL ? left : 0xFFFFFFF0LL;
        if constexpr (DIRECT) {
            const u32x4 d = {(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)) & 0xFFFFu,
                             (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)bytes), 0x00020000u};
            const uint32_t to = (uint32_t)__builtin_amdgcn_readfirstlane(
                (int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds + (int)(threadIdx.x >> 6) * EACH * 1024);
            // (in these terms, and not as the builtin, because the compiler would have the next read of any tile wait for it)
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(to + i * 1024), "v"(from[i]), "s"(d) : "memory");
        } else {
            const Buffer b = buffer_at(reinterpret_cast<const void *>(at), bytes);
#pragma unroll
            for (int i = 0; i < EACH; ++i) held[i] = load16(b, from[i]);
        }
    }
    __device__ __forceinline__ void land(char *lds) const
    {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) *reinterpret_cast<u32x4 *>(lds + vector(i) / VECTORS * kPitch<T, D> + vector(i) % VECTORS * 16) = held[i];
        }
    }
    __device__ __forceinline__ static void landed()
    {
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        __syncthreads();
    }
};

// 32 rows of the wave, as the second operand of `dots`: vector c of lane l is row l % 32, bytes 32 c + 16 (l / 32) and on
template <typename T, int D>
struct Own {
    static constexpr int VECTORS = D / kPerVector<T> / 2;
    u32x4 x[VECTORS];

    __device__ __forceinline__ void load(const T *head, int64_t row, int first, int end, int dim)
    {
        const Buffer b = rows_from(head, row, first, min(end - first, kOwn), dim);
        const int lane = threadIdx.x & 63, r = lane & 31;
#pragma unroll
        for (int c = 0; c < VECTORS; ++c) {
            const int n = 2 * c + (lane >> 5);
            x[c] = load16(b, n * kPerVector<T> < dim ? r * ((int)row * (int)sizeof(T)) + n * 16 : kNowhere);
        }
    }
    // Waits for the rows here.  Left to their first use, inside the loop over tiles, the wait would be for the tiles' loads too.
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int c = 0; c < VECTORS; ++c) asm volatile("" : "+v"(x[c]));
    }
};

__device__ __forceinline__ f32x16 zeros16()
{
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}
// which of 32 rows a lane's element r is
__device__ __forceinline__ int row_of(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }

template <typename T> __device__ __forceinline__ f32x16 multiply16(u32x4 a, u32x4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 multiply16<uint16_t>(u32x4 a, u32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 multiply16<float>(u32x4 a, u32x4 b, f32x16 c)
{
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], c, 0, 0, 0);
    return c;
}

// s of 32 rows of the tile, from row `first` on, and the wave's own
template <typename T, int D>
__device__ __forceinline__ f32x16 dots(const char *tile, int first, const Own<T, D> &own)
{
    const int lane = threadIdx.x & 63;
    const char *at = tile + (first + (lane & 31)) * kPitch<T, D>;
    const int turn = turn_of<T, D>(lane & 31);
    f32x16 s = zeros16();
#pragma unroll
    for (int c = 0; c < Own<T, D>::VECTORS; ++c) s = multiply16<T>(*reinterpret_cast<const u32x4 *>(at + ((2 * c + (lane >> 5)) ^ turn) * 16), own.x[c], s);
    return s;
}

// the same with the wave's own rows in LDS too, from `own` on
template <typename T, int D>
__device__ __forceinline__ f32x16 dots_of(const char *tile, int first, const char *own)
{
    const int lane = threadIdx.x & 63, at = (lane & 31) * kPitch<T, D>, turn = turn_of<T, D>(lane & 31);
    f32x16 s = zeros16();
#pragma unroll
    for (int c = 0; c < Own<T, D>::VECTORS; ++c) {
        const int vector = at + ((2 * c + (lane >> 5)) ^ turn) * 16;
        s = multiply16<T>(*reinterpret_cast<const u32x4 *>(tile + first * kPitch<T, D> + vector), *reinterpret_cast<const u32x4 *>(own + vector), s);
    }
    return s;
}

// both halves of a tile, whose products do not wait for one another; fp32, where products are what takes the time: as many as `halves`
template <typename T, int D>
__device__ __forceinline__ void dots2(const char *tile, const Own<T, D> &own, f32x16 (&s)[2], int halves)
{
    if constexpr (sizeof(T) == 4) {
        s[0] = halves > 0 ? dots<T, D>(tile, 0, own) : zeros16();
        s[1] = halves > 1 ? dots<T, D>(tile, 32, own) : zeros16();
        return;
    }
    const int lane = threadIdx.x & 63;
    const char *at = tile + (lane & 31) * kPitch<T, D>;
    const int turn = turn_of<T, D>(lane & 31);
    s[0] = s[1] = zeros16();
#pragma unroll
    for (int c = 0; c < Own<T, D>::VECTORS; ++c)
#pragma unroll
        for (int n = 0; n < 2; ++n)
            s[n] = multiply16<T>(*reinterpret_cast<const u32x4 *>(at + n * 32 * kPitch<T, D> + ((2 * c + (lane >> 5)) ^ turn) * 16), own.x[c], s[n]);
}

typedef __attribute__((address_space(3))) s16x4 *LdsVector;
__device__ __forceinline__ bf16x8 across(const char *at, const char *and_at)          // four rows' elements of a column, twice
{
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVector)(at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVector)(and_at));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// out[d][o] += sum of tile[t][d] x[t][o] over 32 rows of the tile, from row `first` on.  bf16: x is rounded to bf16 (by 2^-8 of each at
// most, in sums of many of random sign): what the instruction takes; in two parts the product would take twice the time.
template <typename T, int D> __device__ __forceinline__ void sums(const char *tile, int first, const f32x16 &x, f32x16 (&out)[D / 32])
{
    const int lane = threadIdx.x & 63, half = lane >> 5;
    constexpr int P = kPitch<T, D>;
    if constexpr (sizeof(T) == 2) {
        const int row = 4 * half + (lane & 15) / 4, vector = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), turn = turn_of<T, D>(row);
        const char *at = tile + (first + row) * P + (lane & 1) * 8;      // (8 rows on, the turn is another by 2)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const u32x4 b = {bf16_narrow2(x[8 * c], x[8 * c + 1]), bf16_narrow2(x[8 * c + 2], x[8 * c + 3]), bf16_narrow2(x[8 * c + 4], x[8 * c + 5]),
                             bf16_narrow2(x[8 * c + 6], x[8 * c + 7])};
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                out[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    across(at + 16 * c * P + ((4 * i + vector) ^ turn) * 16, at + (16 * c + 8) * P + ((4 * i + vector) ^ turn ^ 2) * 16),
                    __builtin_bit_cast(bf16x8, b), out[i], 0, 0, 0);
        }
    } else {
        const char *at = tile + (first + 4 * half) * P + (lane & 31) * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
                out[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float *>(at + (8 * (r / 4) + r % 4) * P + i * 128), x[r], out[i], 0, 0, 0);
        }
    }
}

// The same for two x of one tile, which is read across once for both.
template <int D> __device__ __forceinline__ void sums_of_two(const char *tile, int first, const f32x16 &x, f32x16 (&out)[D / 32], const f32x16 &y, f32x16 (&more)[D / 32])
{
    const int lane = threadIdx.x & 63, half = lane >> 5;
    constexpr int P = kPitch<uint16_t, D>;
    const int row = 4 * half + (lane & 15) / 4, vector = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), turn = turn_of<uint16_t, D>(row);
    const char *at = tile + (first + row) * P + (lane & 1) * 8;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const u32x4 a = {bf16_narrow2(x[8 * c], x[8 * c + 1]), bf16_narrow2(x[8 * c + 2], x[8 * c + 3]), bf16_narrow2(x[8 * c + 4], x[8 * c + 5]),
                         bf16_narrow2(x[8 * c + 6], x[8 * c + 7])};
        const u32x4 b = {bf16_narrow2(y[8 * c], y[8 * c + 1]), bf16_narrow2(y[8 * c + 2], y[8 * c + 3]), bf16_narrow2(y[8 * c + 4], y[8 * c + 5]),
                         bf16_narrow2(y[8 * c + 6], y[8 * c + 7])};
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const bf16x8 k = across(at + 16 * c * P + ((4 * i + vector) ^ turn) * 16, at + (16 * c + 8) * P + ((4 * i + vector) ^ turn ^ 2) * 16);
            out[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, a), out[i], 0, 0, 0);
            more[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, __builtin_bit_cast(bf16x8, b), more[i], 0, 0, 0);
        }
    }
}

// both halves of a wave hold the same 32 columns
__device__ __forceinline__ float both_max(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float both_sum(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = r[0], b = r[1];
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

// the lane's row of out times `by`, rounded to T; four elements at a time lie beside each other
template <typename T, int D>
__device__ __forceinline__ void store_row(const f32x16 (&out)[D / 32], float by, T *row, int dim)
{
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * i + 8 * g + 4 * half;
            if (d >= dim) continue;
            const float a = out[i][4 * g] * by, b = out[i][4 * g + 1] * by, c = out[i][4 * g + 2] * by, e = out[i][4 * g + 3] * by;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(row + d) = f32x4{a, b, c, e};
            else *reinterpret_cast<u32x2 *>(row + d) = u32x2{bf16_narrow2(a, b), bf16_narrow2(c, e)};
        }
}

template <typename T> __device__ __forceinline__ float widened(T v);
template <> __device__ __forceinline__ float widened<float>(float v) { return v; }
template <> __device__ __forceinline__ float widened<uint16_t>(uint16_t v) { return bf16_widen(v); }

// The head's column of the table, in LDS, and the biases of a tile's distances.  A bucket outside of the table adds nothing.
struct BiasLoad {
    int bucket;

    // distances from first on, counted as in bucket_of
    __device__ __forceinline__ void load(const Attention &a, int first)
    {
        const int t = threadIdx.x, at = first + t;
        bucket = t < kDistances && at >= 0 && at < a.q_tokens + a.k_tokens - 1 ? a.bucket_of[at] : -1;
    }
    __device__ __forceinline__ void store(const Attention &a, const float *column, float *bias) const
    {
        if (threadIdx.x < kDistances) bias[threadIdx.x] = (uint32_t)bucket < (uint32_t)a.buckets ? column[bucket] : 0.0f;
    }
};
template <typename T>
__device__ __forceinline__ void load_column(const Attention &a, int head, float *column)
{
    for (int i = threadIdx.x; i < a.buckets; i += kAttnThreads) column[i] = widened(static_cast<const T *>(a.table)[(int64_t)i * a.q_heads + head]);
}

// The launches.  splits 0: 128 queries a workgroup; above: few queries, the keys shared out over so many workgroups, whose sums meet in parts.
void attention_forward_f32(const Attention &a, void *out, float *stats, float *parts, int splits, hipStream_t st);
void attention_forward_bf16(const Attention &a, void *out, float *stats, float *parts, int splits, hipStream_t st);

struct Gradients {
    const void *dout, *out;
    const float *stats;
    void *dq, *dk, *dv;
    int64_t dq_b, dq_h, dq_t, dk_b, dk_h, dk_t, dk_d, dv_b, dv_h, dv_t;
    float *rows;                             // [3][batch * q_heads * q_tokens]: what p is taken by (two numbers), delta
    float *parts;                            // sums of ds by distance, or NULL
    int64_t part_row;                        // floats of a wave's
    int32_t first_block, blocks;             // of queries: those of one launch, whose sums by distance parts holds
    bool all_rows;                           // the last of these launches, after which the keys' gradients follow
    // workgroups that share the tiles of one block out, and, where that is more than one, their sums: dq [q_splits][batch][q_heads]
    // [q_tokens][head_dim], dk and dv [k_splits][batch][kv_heads][k_tokens][2][head_dim]
    int32_t q_splits, k_splits;
    float *dq_parts, *dk_parts;
};
void attention_backward_f32(const Attention &a, const Gradients &g, hipStream_t st);
void attention_backward_bf16(const Attention &a, const Gradients &g, hipStream_t st);
}  // namespace slimfit
