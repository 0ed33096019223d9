// Attention: the calls' checks and launches, and the small passes around the kernels of attention_forward.hpp and attention_backward.hpp:
// keys that lie transposed are turned into rows first (2 bytes moved for each; the products read rows of either side), and
// the sums of ds by distance that the waves left are added up over batch and queries, then over each bucket's distances, in order.
#include "attention.hpp"

namespace slimfit {
namespace {

constexpr int kTurn = 64;
constexpr int64_t kTurnBytes = (int64_t)256 << 20, kTurnWorkgroups = 2048;      // (`turn_blocks`)
constexpr int kAtOnce = 8;                   // blocks of queries whose sums by distance are under way at a time

// kt (head, dim, tokens) -> k (head, tokens, dim): a workgroup takes 64 tokens of up to 64 elements, 16 bytes a thread in and out.  Rows of dim
// begin on 16 bytes, those of tokens anywhere (8 heads of 96, 4097 tokens: 6.0 us, element by element 9.4).
typedef u32x4 Anywhere __attribute__((aligned(2)));
template <typename T>
__global__ void __launch_bounds__(kAttnThreads) turn_kernel(const T *__restrict__ kt, T *__restrict__ k, int dim, int tokens, int blocks, int columns)
{
    constexpr int E = kPerVector<T>, LINE = kTurn / E, LINES = kAttnThreads / LINE;
    __shared__ T tile[kTurn][kTurn + 4 / sizeof(T)];        // [element][token]: an odd number of banks apart
    const int unit = (int)(blockIdx.x / (unsigned)(blocks * columns)), rest = (int)(blockIdx.x % (unsigned)(blocks * columns));
    const int t0 = rest / columns * kTurn, d0 = rest % columns * kTurn;
    const T *const from = kt + (int64_t)unit * dim * tokens;
    T *const to = k + (int64_t)unit * dim * tokens;
    const int x = threadIdx.x % LINE * E, y = threadIdx.x / LINE;
    u32x4 v[kTurn / LINES];
#pragma unroll
    for (int i = 0; i < kTurn / LINES; ++i) {
        const int d = d0 + y + i * LINES;
        v[i] = u32x4{0u, 0u, 0u, 0u};
        if (d < dim && t0 + x + E <= tokens) v[i] = *reinterpret_cast<const Anywhere *>(from + (int64_t)d * tokens + t0 + x);
    }
#pragma unroll
    for (int i = 0; i < kTurn / LINES; ++i) {
        const int d = d0 + y + i * LINES;
        if (d >= dim || t0 + x >= tokens) continue;
        if (t0 + x + E > tokens) {                          // the last few
            for (int e = 0; t0 + x + e < tokens; ++e) tile[y + i * LINES][x + e] = from[(int64_t)d * tokens + t0 + x + e];
            continue;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t w = v[i][e * (int)sizeof(T) / 4];
            if constexpr (sizeof(T) == 4) tile[y + i * LINES][x + e] = __builtin_bit_cast(float, w);
            else tile[y + i * LINES][x + e] = (T)(w >> (16 * (e & 1)));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTurn; i += LINES) {
        if (t0 + y + i >= tokens || d0 + x >= dim) continue;
        u32x4 line;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (sizeof(T) == 4) line[w] = __builtin_bit_cast(uint32_t, tile[x + w][y + i]);
            else line[w] = (uint32_t)tile[x + 2 * w][y + i] | (uint32_t)tile[x + 2 * w + 1][y + i] << 16;
        }
        *reinterpret_cast<u32x4 *>(to + (int64_t)(t0 + y + i) * dim + d0 + x) = line;
    }
}

// Sums of ds by distance over `each` of `blocks` blocks of 128 queries from the first_block-th on (and shares of their keys) of all sequences: blockIdx.z has its
// share, in order, added to that of the blocks before.  What a wave did not
// write is past its descriptor's end: 0, with no branch that a load would wait at (512 tokens: 11.6 us with branches, 5.0 without).
__global__ void __launch_bounds__(kWave) distances_kernel(Attention a, const float *__restrict__ parts, int64_t part_row, int first_block, int blocks, int splits, int each, float *__restrict__ sums)
{
    const int all = a.q_tokens + a.k_tokens - 1, head = blockIdx.y, at = (int)(blockIdx.x * kWave + threadIdx.x);
    const int end = min(a.batch * blocks * splits, ((int)blockIdx.z + 1) * each);
    float *const to = sums + ((int64_t)blockIdx.z * a.q_heads + head) * all + at;
    double sum = first_block > 0 && at < all ? (double)*to : 0.0;
    for (int n0 = (int)blockIdx.z * each; n0 < end; n0 += kAtOnce) {
        float x[kAtOnce][kAttnWaves];
        const int keys = keys_of(a, min(n0 + (int)(threadIdx.x % kAtOnce), end - 1) / splits / blocks);                 // a block's a lane
#pragma unroll
        for (int m = 0; m < kAtOnce; ++m) {
            const int n = min(n0 + m, end - 1), split = n % splits, b = n / splits / blocks, block = n / splits % blocks;
            const int q0 = (first_block + block) * kBlock, tiles = key_tiles(a, q0, __builtin_amdgcn_readlane(keys, m)), t0 = first_of(tiles, split, splits);
            const int written = (first_of(tiles, split + 1, splits) - t0) * kTile + kOwn;
            const float *const of = parts + ((((int64_t)b * a.q_heads + head) * blocks + block) * splits + split) * kAttnWaves * part_row;
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w) {
                const int place = at - (a.q_tokens - 1) + q0 + w * kOwn + kOwn - 1 - t0 * kTile;
                const Buffer row = buffer_at(of + w * part_row, n0 + m < end ? (int64_t)written * 4 : 0);
                // (a sum of an offset below 0 and a constant would be past the end even where it is not)
                x[m][w] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(row, place < 0 ? kNowhere : place * 4, 0, 0));
            }
        }
#pragma unroll
        for (int m = 0; m < kAtOnce; ++m)
#pragma unroll
            for (int w = 0; w < kAttnWaves; ++w) sum += (double)x[m][w];
    }
    if (at < all) *to = (float)sum;
}

// a workgroup for each bucket and head
template <typename T>
__global__ void __launch_bounds__(kAttnThreads) buckets_kernel(Attention a, const float *__restrict__ sums, int shares, T *__restrict__ dtable)
{
    __shared__ double part[kAttnWaves];
    const int all = a.q_tokens + a.k_tokens - 1, bucket = blockIdx.x, head = blockIdx.y;
    double sum = 0.0;
    const int64_t apart = (int64_t)a.q_heads * all;
    const float *const from = sums + (int64_t)head * all;
    for (int at0 = 0; at0 < (shares > 0 ? all : 0); at0 += kAttnThreads) {      // (no sums otherwise)
        const int at = at0 + (int)threadIdx.x;
        const bool in = at < all && a.bucket_of[min(at, all - 1)] == bucket;
        if (__builtin_amdgcn_ballot_w64(in) == 0u) continue;
        for (int z0 = 0; z0 < shares; z0 += kAtOnce) {      // (as above: what is not the bucket's is past the end)
            float x[kAtOnce];
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z)
                x[z] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(buffer_at(from + (z0 + z) * apart, z0 + z < shares ? (int64_t)all * 4 : 0), in ? at * 4 : kNowhere, 0, 0));
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) sum += (double)x[z];
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, kWave);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x > 0) return;
    const float x = (float)(((part[0] + part[1]) + part[2]) + part[3]);
    if constexpr (sizeof(T) == 4) dtable[(int64_t)bucket * a.q_heads + head] = x;
    else dtable[(int64_t)bucket * a.q_heads + head] = (T)bf16_narrow(x);
}

// Where tiles of a block were shared out: dq, dk and dv from the shares' sums, in order, four elements of a row a thread.  (Transposed keys'
// gradients by element, tokens beside each other.)
template <typename T> __device__ __forceinline__ void store4(T *to, f32x4 x)
{
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(to) = x;
    else *reinterpret_cast<u32x2 *>(to) = u32x2{bf16_narrow2(x[0], x[1]), bf16_narrow2(x[2], x[3])};
}
template <typename T>
__global__ void __launch_bounds__(kAttnThreads) shares_kernel(Attention a, Gradients g)
{
    const int vectors = a.head_dim / 4;
    const int64_t q_rows = g.q_splits > 1 ? (int64_t)a.batch * a.q_heads * a.q_tokens : 0, k_rows = g.k_splits > 1 ? (int64_t)a.batch * a.kv_heads * a.k_tokens : 0;
    int64_t n = (int64_t)blockIdx.x * kAttnThreads + threadIdx.x;
    const bool query = n < q_rows * vectors;
    if (!query && (n -= q_rows * vectors) >= 2 * k_rows * vectors) return;
    const int tokens = query ? a.q_tokens : a.k_tokens, heads = query ? a.q_heads : a.kv_heads, width = query ? vectors : 2 * vectors;
    int64_t row;
    int v;
    if (!query && g.dk_d != 1) {
        const int64_t line = n / tokens;                    // of a pair's vectors
        row = line / width * tokens + n % tokens;
        v = (int)(line % width);
    } else {
        row = n / width;
        v = (int)(n % width);
    }
    const float *from = (query ? g.dq_parts : g.dk_parts) + (row * width + v) * 4;
    const int64_t step = (query ? q_rows : k_rows) * width * 4;
    f32x4 sum = *reinterpret_cast<const f32x4 *>(from);
    for (int s = 1; s < (query ? g.q_splits : g.k_splits); ++s) sum += *reinterpret_cast<const f32x4 *>(from + s * step);
    const int64_t pair = row / tokens, token = row % tokens, batch = pair / heads, head = pair % heads;
    if (query) {
        store4(static_cast<T *>(g.dq) + batch * g.dq_b + head * g.dq_h + token * g.dq_t + v * 4, sum);
    } else if (v >= vectors) {
        store4(static_cast<T *>(g.dv) + batch * g.dv_b + head * g.dv_h + token * g.dv_t + (v - vectors) * 4, sum);
    } else if (g.dk_d == 1) {
        store4(static_cast<T *>(g.dk) + batch * g.dk_b + head * g.dk_h + token * g.dk_t + v * 4, sum);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            T *const to = static_cast<T *>(g.dk) + batch * g.dk_b + head * g.dk_h + token * g.dk_t + (v * 4 + e) * g.dk_d;
            if constexpr (sizeof(T) == 4) *to = sum[e];
            else *to = (T)bf16_narrow(sum[e]);
        }
    }
}

struct Sizes {
    int32_t dt, layout;
    int64_t batch;
    int32_t q_tokens, k_tokens, q_heads, kv_heads, head_dim, buckets;
    size_t e() const { return dtype_size(dt); }
    int64_t q_count() const { return batch * q_tokens * q_heads * head_dim; }
    int64_t k_count() const { return batch * k_tokens * kv_heads * head_dim; }
};

size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

int32_t check_sizes(const Sizes &z)
{
    if (!dtype_ok(z.dt) || (z.layout != SLIMFIT_HEADS_ROWS && z.layout != SLIMFIT_HEADS_APART)) return SLIMFIT_ERR_INVALID_ARG;
    if (z.batch < 0 || z.q_tokens < 0 || z.k_tokens < 0 || z.q_heads < 1 || z.kv_heads < 1 || z.q_heads % z.kv_heads != 0 || z.head_dim < 1 || z.buckets < 0)
        return SLIMFIT_ERR_INVALID_ARG;
    if (z.head_dim % (16 / (int)z.e()) != 0 || z.head_dim > kMostHeadDim || z.buckets > kMostBuckets || z.q_heads > (1 << 15)) return SLIMFIT_ERR_UNSUPPORTED;
    if (z.q_tokens > (1 << 28) || z.k_tokens > (1 << 28) || z.batch > (1 << 24)) return SLIMFIT_ERR_UNSUPPORTED;
    const int64_t blocks = ((int64_t)(z.q_tokens > z.k_tokens ? z.q_tokens : z.k_tokens) + kBlock - 1) / kBlock;
    // (the turned keys take up to four workgroups for each of these)
    if (z.batch * z.q_heads * (blocks > 0 ? blocks : 1) >= ((int64_t)1 << 22)) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

bool turned(const Sizes &z) { return z.layout == SLIMFIT_HEADS_APART && z.batch > 0 && z.k_tokens > 0 && z.q_tokens > 0; }
size_t turned_bytes(const Sizes &z) { return turned(z) ? rounded((size_t)z.k_count() * z.e()) : 0; }
int q_blocks(const Sizes &z) { return (z.q_tokens + kBlock - 1) / kBlock; }
// Backward: how many workgroups share the tiles of a block's other side out where blocks do not fill the card; their sums meet in memory,
// added up in order by one more launch.  (us of the backward pass in one share, so; T tokens, a head each T / 128 blocks)
//   fp32, whose tiles take longest: as many as make the rounds of 256 workgroups times the tiles of one, and one more for its start, the least, up
//   to 320 blocks.  Heads of 128: 1 x 200 120, 53; 6 x 512 249, 69; 1 x 1400 638, 91; 6 x 1400 655, 270; 16 x 1400 causal 695, 428; 24 x 1400 1310,
//   1010; 4 x 4097 2450, 1210.  Of 32: 1 x 200 37, 21; 40 x 200 38, 32; 6 x 1400 187, 85.  (With 384 blocks of 128, 96 x 512, all 508, 475, but causal
//   312, 384; with 792, 24 x 4097, all 7540, 6490, but causal 3525, 3924.)
//   bf16, where the queries' shares each go over all keys for delta: up to as many blocks as four for a tile: heads of 128: 1 x 512 56, 39; 6 x 512 57,
//   48; 6 x 1400 139, 102; of 32: 1 x 512 22, 20; 1 x 1400 53, 33; 6 x 1400 56, 49; but 16 x 512 24, 28; 40 x 300 20, 26.
int splits_of(const Sizes &z, int64_t workgroups, int64_t tiles)
{
    if (workgroups == 0) return 1;
    if (z.dt == SLIMFIT_BF16) {
        if (tiles < 8 || workgroups > 4 * tiles) return 1;
        const int64_t splits = 256 / workgroups < tiles / 2 ? 256 / workgroups : tiles / 2;
        return splits < 1 ? 1 : splits > kMostSplits ? kMostSplits : (int)splits;
    }
    int best = 1;
    int64_t least = 0;
    for (int s = 1; s <= kMostSplits && s <= tiles && (s == 1 || workgroups <= 320); ++s) {
        const int64_t cost = 8 * ((workgroups * s + 255) / 256) * ((tiles + s - 1) / s + 1) + s;
        if (s == 1 || cost < least) {
            best = s;
            least = cost;
        }
    }
    return best;
}
int query_splits(const Sizes &z) { return splits_of(z, z.batch * z.q_heads * q_blocks(z), ((int64_t)z.k_tokens + kTile - 1) / kTile); }
int key_splits(const Sizes &z)
{
    return splits_of(z, z.batch * z.kv_heads * ((z.k_tokens + kBlock - 1) / kBlock), (int64_t)(z.q_heads / z.kv_heads) * ((z.q_tokens + kTile - 1) / kTile));
}
// floats that a wave has for its sums by distance: those of the largest share of a block's tiles, and 32 more
int64_t part_row(const Sizes &z)
{
    const int64_t tiles = ((int64_t)z.k_tokens + kTile - 1) / kTile, splits = query_splits(z);
    return ((tiles + splits - 1) / splits + 1) * kTile;
}
// Blocks of queries whose sums by distance are held at a time, a launch each: kTurnBytes of these or, at long rows, as many as make kTurnWorkgroups,
// so that they take memory by the keys and not by the pairs.  (Blocks whose tiles are shared out are fewer.)  16 x 4096 x 4096, 16 heads of 64: three
// launches 7080 us, one 7085; with no kTurnBytes 300 x 512 x 512, 12 heads, is in four, 2221 us for 1944.
int turn_blocks(const Sizes &z)
{
    if (z.batch == 0 || q_blocks(z) == 0) return q_blocks(z);
    const int64_t units = z.batch * z.q_heads, by_bytes = kTurnBytes / (units * kAttnWaves * part_row(z) * 4), by_workgroups = kTurnWorkgroups / units;
    const int64_t most = by_bytes > by_workgroups ? by_bytes : by_workgroups;
    return most < 1 ? 1 : most < q_blocks(z) ? (int)most : q_blocks(z);
}
// blocks of queries that one share of the sums by distance adds up (16 x 512, 12 heads: 64 in one share 57 us, 8 each 6.6), and the shares
int64_t share_of(const Sizes &z)
{
    const int64_t all = z.batch * turn_blocks(z) * query_splits(z);
    return all <= 8 * 32 ? 8 : (all + 31) / 32;
}
int64_t shares_of(const Sizes &z) { return (z.batch * turn_blocks(z) * query_splits(z) + share_of(z) - 1) / share_of(z); }

// How many workgroups share a sequence's keys out, or 0: 128 queries of a head a workgroup.  (us with those, with few queries, on the same operands again and again)
//   bf16, up to 16 queries: 16 x 4096 keys, 32 heads on 8 by 128: 1 query 121, 48; 16 132, 63; 32 139, 120; 64 142, 243;
//         64 x 1024, 8 heads of 64: 1 24.5, 25.4; 16 25.3, 25.7; 64 25.5, 48.5.
//   fp32, where padded queries cost products, up to 64: the first 1 1146, 137; 64 1153, 926; the second 1 137, 48; 64 142, 105.
//   Any where there are few workgroups otherwise and keys are many: bf16, 1 x 4096, 32 heads on 8 by 128: 128 queries 95, 46; 8 x 1024,
//         12 heads of 64: 64 queries 18.6, 13.1; of 128 keys 5.7, 6.8.  fp32, whose products are a wave's time, from 128 keys on: 40 heads of
//         64, 128 x 128 13.8, 9.6; 300 x 300 27.9, 23.2; 16 heads of 128, 300 x 300 51.4, 27.6; but 64 heads, 192 workgroups otherwise, 54.7, 79.0.
// A workgroup for each compute unit is enough (16 x 4096 and 1 query: 256 workgroups 48, 512 54, 1024 60), but for fp32 heads of up
// to 64, two of which fit one (8 x 4096, 12 heads: 65, 47, 55).
int few_splits(const Sizes &z)
{
    if (z.batch == 0 || z.q_tokens == 0 || z.k_tokens == 0) return 0;
    const int64_t others = z.batch * z.q_heads * q_blocks(z);
    if (z.q_tokens > (z.dt == SLIMFIT_BF16 ? 16 : 64) && (others > 128 || z.k_tokens < (z.dt == SLIMFIT_BF16 ? 512 : 128))) return 0;
    const int64_t rows = (int64_t)(z.q_heads / z.kv_heads) * z.q_tokens, blocks = z.batch * z.kv_heads * ((rows + kOwn - 1) / kOwn);
    const int64_t tiles = (z.k_tokens + kFewTile - 1) / kFewTile;
    int64_t splits = (z.dt == SLIMFIT_F32 && z.head_dim <= 64 ? 512 : 256) / blocks;
    if (splits > tiles) splits = tiles;
    if (splits > kMostSplits) splits = kMostSplits;
    return splits < 1 ? 1 : (int)splits;
}
size_t part_bytes(const Sizes &z)
{
    const int splits = few_splits(z);
    return splits > 1 ? rounded((size_t)(z.batch * z.q_heads) * (size_t)z.q_tokens * (size_t)splits * ((size_t)z.head_dim + 2) * 4) : 0;
}

struct BackwardPlaces {
    size_t rows, parts, sums, dq, dk, bytes;
    BackwardPlaces(const Sizes &z, bool table)
    {
        rows = turned_bytes(z);
        parts = rows + rounded((size_t)(z.batch * z.q_heads) * (size_t)z.q_tokens * 12);
        sums = parts + (table ? rounded((size_t)(z.batch * z.q_heads) * (size_t)(turn_blocks(z) * query_splits(z)) * kAttnWaves * (size_t)part_row(z) * 4) : 0);
        dq = sums + (table ? rounded((size_t)shares_of(z) * (size_t)z.q_heads * ((size_t)z.q_tokens + (size_t)z.k_tokens) * 4) : 0);
        dk = dq + (query_splits(z) > 1 ? rounded((size_t)query_splits(z) * (size_t)z.q_count() * 4) : 0);
        bytes = dk + (key_splits(z) > 1 ? rounded((size_t)key_splits(z) * (size_t)z.k_count() * 8) : 0);
    }
};

// One operand's memory: `rows` rows of `width` bytes, `apart` bytes from one to the next.
struct Span {
    const void *at;
    size_t rows, width, apart;
    size_t bytes() const { return rows == 0 ? 0 : (rows - 1) * apart + width; }
};
bool share(const Span &a, const Span &b)
{
    if (a.bytes() == 0 || b.bytes() == 0 || !meet(a.at, a.bytes(), b.at, b.bytes())) return false;
    if (a.apart != b.apart) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);     // columns of the same rows
    const size_t off = y >= x ? (size_t)(y - x) % a.apart : a.apart - 1 - (size_t)(x - y - 1) % a.apart;
    return off < a.width || a.apart - off < b.width;
}

// q, k, v or their gradients
Operand operand_of(const void *at, const Sizes &z, int which, int64_t row)
{
    const int64_t heads = which == 0 ? z.q_heads : z.kv_heads, tokens = which == 0 ? z.q_tokens : z.k_tokens, D = z.head_dim;
    if (z.layout == SLIMFIT_HEADS_ROWS) return {at, tokens * row, D, row};
    return {at, heads * tokens * D, tokens * D, D};
}
Span span_of(const void *at, const Sizes &z, int which, int64_t row)
{
    const size_t heads = (size_t)(which == 0 ? z.q_heads : z.kv_heads), tokens = (size_t)(which == 0 ? z.q_tokens : z.k_tokens), D = (size_t)z.head_dim;
    if (z.layout == SLIMFIT_HEADS_ROWS) return {at, (size_t)z.batch * tokens, heads * D * z.e(), (size_t)row * z.e()};
    const size_t all = (size_t)z.batch * heads * tokens * D * z.e();
    return {at, all > 0 ? 1u : 0u, all, all};
}
Span flat(const void *at, size_t bytes) { return {at, bytes > 0 ? 1u : 0u, bytes, bytes}; }

int32_t check_rows(const Sizes &z, int64_t q_row, int64_t k_row, int64_t v_row)
{
    if (z.layout != SLIMFIT_HEADS_ROWS) return SLIMFIT_OK;
    const int64_t per = 16 / (int64_t)z.e(), kv = (int64_t)z.kv_heads * z.head_dim;
    if (q_row < (int64_t)z.q_heads * z.head_dim || k_row < kv || v_row < kv) return SLIMFIT_ERR_INVALID_ARG;
    if (q_row % per != 0 || k_row % per != 0 || v_row % per != 0) return SLIMFIT_ERR_ALIGNMENT;
    return q_row > (1 << 20) || k_row > (1 << 20) || v_row > (1 << 20) ? SLIMFIT_ERR_UNSUPPORTED : SLIMFIT_OK;
}

// the spans' pointers, alignment (NULL where there is nothing is fine) and that no output shares memory with anything
int32_t check_spans(const Span *in, int n_in, const Span *out, int n_out)
{
    for (int i = 0; i < n_in + n_out; ++i) {
        const Span &s = i < n_in ? in[i] : out[i - n_in];
        if (s.bytes() > 0 && !s.at) return SLIMFIT_ERR_INVALID_ARG;
    }
    for (int i = 0; i < n_in + n_out; ++i)
        if (!aligned_to(i < n_in ? in[i].at : out[i - n_in].at, 16)) return SLIMFIT_ERR_ALIGNMENT;
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (share(out[i], in[j])) return SLIMFIT_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (share(out[i], out[j])) return SLIMFIT_ERR_INVALID_ARG;
    }
    return SLIMFIT_OK;
}
int32_t check_ranges(const Span *s, int n)
{
    int32_t rc;
    for (int i = 0; i < n; ++i)
        if ((rc = check_device_range(s[i].at, s[i].bytes())) != SLIMFIT_OK) return rc;
    return SLIMFIT_OK;
}

int32_t check_others(const Sizes &z, float scale, const int32_t *lengths, const void *table, const int32_t *bucket_of)
{
    if (!(scale > 0.0f) || scale >= 0x1p127f) return SLIMFIT_ERR_INVALID_ARG;     // (scale log2 e has to be a number)
    if (table && (z.buckets < 1 || (!bucket_of && z.q_tokens > 0 && z.k_tokens > 0))) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(lengths, 4) || !aligned_to(table, z.e()) || (table && !aligned_to(bucket_of, 4))) return SLIMFIT_ERR_ALIGNMENT;
    return SLIMFIT_OK;
}
int32_t check_other_ranges(const Sizes &z, const int32_t *lengths, const void *table, const int32_t *bucket_of)
{
    int32_t rc;
    if (lengths && (rc = check_device_range(lengths, (size_t)z.batch * 4)) != SLIMFIT_OK) return rc;
    if (!table) return SLIMFIT_OK;
    if ((rc = check_device_range(table, (size_t)z.buckets * (size_t)z.q_heads * z.e())) != SLIMFIT_OK) return rc;
    return z.q_tokens > 0 && z.k_tokens > 0 ? check_device_range(bucket_of, ((size_t)z.q_tokens + (size_t)z.k_tokens - 1) * 4) : SLIMFIT_OK;
}
// what a call reads beside its operands
struct Others {
    Span s[3];
    Others(const Sizes &z, const int32_t *lengths, const void *table, const int32_t *bucket_of)
        : s{flat(lengths, lengths ? (size_t)z.batch * 4 : 0), flat(table, table ? (size_t)z.buckets * (size_t)z.q_heads * z.e() : 0),
            flat(bucket_of, table && z.q_tokens > 0 && z.k_tokens > 0 ? ((size_t)z.q_tokens + (size_t)z.k_tokens - 1) * 4 : 0)}
    {
    }
};
bool any_share(const Span *a, int n_a, const Span *b, int n_b)
{
    for (int i = 0; i < n_a; ++i)
        for (int j = 0; j < n_b; ++j)
            if (share(a[i], b[j])) return true;
    return false;
}
// the workspace, which shares memory with nothing else of the call
int32_t check_workspace(size_t need, const void *ws, size_t bytes, const Span *in, int n_in, const Span *out, int n_out, const Others &others)
{
    if (need == 0) return SLIMFIT_OK;
    if (!ws || bytes < need) return SLIMFIT_ERR_WORKSPACE;
    if (!aligned_to(ws, 16)) return SLIMFIT_ERR_ALIGNMENT;
    const Span w = flat(ws, need);
    if (any_share(&w, 1, in, n_in) || any_share(&w, 1, out, n_out) || any_share(&w, 1, others.s, 3)) return SLIMFIT_ERR_INVALID_ARG;
    return check_device_range(ws, need);
}

void turn_keys(const Sizes &z, const void *kt, void *k, hipStream_t st)
{
    const int blocks = (z.k_tokens + kTurn - 1) / kTurn, columns = (z.head_dim + kTurn - 1) / kTurn;
    const unsigned grid = (unsigned)(z.batch * z.kv_heads * blocks * columns);
    if (z.dt == SLIMFIT_F32) launch(turn_kernel<float>, grid, kAttnThreads, 0, st, static_cast<const float *>(kt), static_cast<float *>(k), z.head_dim, z.k_tokens, blocks, columns);
    else launch(turn_kernel<uint16_t>, grid, kAttnThreads, 0, st, static_cast<const uint16_t *>(kt), static_cast<uint16_t *>(k), z.head_dim, z.k_tokens, blocks, columns);
}

Attention attention_of(const Sizes &z, const void *q, const void *k, const void *v, int64_t q_row, int64_t k_row, int64_t v_row, float scale, int32_t causal,
                       const int32_t *lengths, const void *table, const int32_t *bucket_of)
{
    return {operand_of(q, z, 0, q_row), operand_of(k, z, 1, k_row), operand_of(v, z, 1, v_row), (int32_t)z.batch, z.q_tokens, z.k_tokens, z.q_heads, z.kv_heads,
            z.head_dim, causal != 0, table ? z.buckets : 0, scale, lengths, table, bucket_of};
}

}  // namespace
}  // namespace slimfit

using namespace slimfit;

extern "C" int32_t slimfit_attention_workspace(int32_t dt, int32_t layout, int64_t batch, int32_t q_tokens, int32_t k_tokens, int32_t q_heads, int32_t kv_heads,
                                               int32_t head_dim, int32_t with_dtable, int32_t backward, size_t *bytes)
{
    const Sizes z = {dt, layout, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, 0};
    const int32_t rc = check_sizes(z);
    if (rc != SLIMFIT_OK) return rc;
    if (!bytes) return SLIMFIT_ERR_INVALID_ARG;
    *bytes = backward ? BackwardPlaces(z, with_dtable != 0).bytes : turned_bytes(z) + part_bytes(z);
    return SLIMFIT_OK;
}

extern "C" int32_t slimfit_attention_forward(const void *q, const void *k, const void *v, int32_t dt, int32_t layout, int64_t q_row, int64_t k_row, int64_t v_row,
                                             int64_t batch, int32_t q_tokens, int32_t k_tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale,
                                             int32_t causal, const int32_t *lengths, const void *table, int32_t buckets, const int32_t *bucket_of, void *out,
                                             float *stats, void *workspace, size_t workspace_bytes, void *stream)
{
    StreamScope capture_aware(stream);
    const Sizes z = {dt, layout, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, table ? buckets : 0};
    int32_t rc = check_sizes(z);
    if (rc != SLIMFIT_OK || (rc = check_rows(z, q_row, k_row, v_row)) != SLIMFIT_OK) return rc;
    if ((rc = check_others(z, scale, lengths, table, bucket_of)) != SLIMFIT_OK) return rc;
    if (batch == 0 || q_tokens == 0) return SLIMFIT_OK;
    const Span in[] = {span_of(q, z, 0, q_row), span_of(k, z, 1, k_row), span_of(v, z, 1, v_row)};
    const Span to[] = {flat(out, (size_t)z.q_count() * z.e()), flat(stats, (size_t)(batch * q_heads) * (size_t)q_tokens * 8)};
    const Others others(z, lengths, table, bucket_of);
    if ((rc = check_spans(in, 3, to, 2)) != SLIMFIT_OK) return rc;
    if (any_share(to, 2, others.s, 3)) return SLIMFIT_ERR_INVALID_ARG;
    const size_t need = turned_bytes(z) + part_bytes(z);
    if ((rc = check_workspace(need, workspace, workspace_bytes, in, 3, to, 2, others)) != SLIMFIT_OK) return rc;
    if ((rc = check_ranges(in, 3)) != SLIMFIT_OK || (rc = check_ranges(to, 2)) != SLIMFIT_OK) return rc;
    if ((rc = check_other_ranges(z, lengths, table, bucket_of)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (turned(z)) {
        turn_keys(z, k, workspace, st);
        k = workspace;
    }
    const Attention a = attention_of(z, q, k, v, q_row, k_row, v_row, scale, causal, lengths, k_tokens > 0 ? table : nullptr, bucket_of);
    float *const parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + turned_bytes(z));
    if (dt == SLIMFIT_BF16) attention_forward_bf16(a, out, stats, parts, few_splits(z), st);
    else attention_forward_f32(a, out, stats, parts, few_splits(z), st);
    return launch_status();
}

extern "C" int32_t slimfit_attention_backward(const void *dout, const void *q, const void *k, const void *v, int32_t dt, int32_t layout, int64_t q_row,
                                              int64_t k_row, int64_t v_row, int64_t batch, int32_t q_tokens, int32_t k_tokens, int32_t q_heads, int32_t kv_heads,
                                              int32_t head_dim, float scale, int32_t causal, const int32_t *lengths, const void *table, int32_t buckets,
                                              const int32_t *bucket_of, const void *out, const float *stats, void *dq, void *dk, void *dv, int64_t dq_row,
                                              int64_t dk_row, int64_t dv_row, void *dtable, void *workspace, size_t workspace_bytes, void *stream)
{
    StreamScope capture_aware(stream);
    const Sizes z = {dt, layout, batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, table ? buckets : 0};
    int32_t rc = check_sizes(z);
    if (rc != SLIMFIT_OK || (rc = check_rows(z, q_row, k_row, v_row)) != SLIMFIT_OK || (rc = check_rows(z, dq_row, dk_row, dv_row)) != SLIMFIT_OK) return rc;
    if ((rc = check_others(z, scale, lengths, table, bucket_of)) != SLIMFIT_OK) return rc;
    if (dtable && !table) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(dtable, z.e())) return SLIMFIT_ERR_ALIGNMENT;
    const size_t q_bytes = (size_t)z.q_count() * z.e(), table_bytes = dtable ? (size_t)buckets * (size_t)q_heads * z.e() : 0;
    const Span in[] = {span_of(q, z, 0, q_row), span_of(k, z, 1, k_row), span_of(v, z, 1, v_row), flat(dout, q_bytes), flat(out, q_bytes),
                       flat(stats, (size_t)(batch * q_heads) * (size_t)q_tokens * 8)};
    const Span to[] = {span_of(dq, z, 0, dq_row), span_of(dk, z, 1, dk_row), span_of(dv, z, 1, dv_row), flat(dtable, table_bytes)};
    const Others others(z, lengths, table, bucket_of);
    if ((rc = check_spans(in, 6, to, 3)) != SLIMFIT_OK) return rc;
    if (any_share(to + 3, 1, in, 6) || any_share(to + 3, 1, to, 3) || any_share(to, 4, others.s, 3)) return SLIMFIT_ERR_INVALID_ARG;
    const BackwardPlaces at(z, dtable != nullptr);
    if ((rc = check_workspace(at.bytes, workspace, workspace_bytes, in, 6, to, 4, others)) != SLIMFIT_OK) return rc;
    if ((rc = check_ranges(in, 6)) != SLIMFIT_OK || (rc = check_ranges(to, 3)) != SLIMFIT_OK) return rc;
    if ((rc = check_other_ranges(z, lengths, table, bucket_of)) != SLIMFIT_OK || (rc = check_device_range(dtable, table_bytes)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *const ws = static_cast<char *>(workspace);
    if (turned(z)) {
        turn_keys(z, k, ws, st);
        k = ws;
    }
    const bool pairs = batch > 0 && q_tokens > 0 && k_tokens > 0;
    const Attention a = attention_of(z, q, k, v, q_row, k_row, v_row, scale, causal, lengths, pairs ? table : nullptr, bucket_of);
    const Operand oq = operand_of(dq, z, 0, dq_row), ok = operand_of(dk, z, 1, dk_row), ov = operand_of(dv, z, 1, dv_row);
    const bool across = layout == SLIMFIT_HEADS_APART;      // dk lies transposed too: tokens beside each other
    float *const parts = dtable && pairs ? reinterpret_cast<float *>(ws + at.parts) : nullptr;
    Gradients g = {dout, out, stats, dq, dk, dv, oq.b, oq.h, oq.t, ok.b, ok.h, across ? 1 : ok.t, across ? k_tokens : 1, ov.b, ov.h, ov.t,
                   reinterpret_cast<float *>(ws + at.rows), parts, part_row(z), 0, 0, false, query_splits(z), key_splits(z), reinterpret_cast<float *>(ws + at.dq),
                   reinterpret_cast<float *>(ws + at.dk)};
    float *const sums = reinterpret_cast<float *>(ws + at.sums);
    const int all = q_tokens + k_tokens - 1, shares = parts ? (int)shares_of(z) : 0, turn = parts ? turn_blocks(z) : q_blocks(z);
    do {
        g.blocks = q_blocks(z) - g.first_block < turn ? q_blocks(z) - g.first_block : turn;
        g.all_rows = g.first_block + g.blocks == q_blocks(z);
        if (dt == SLIMFIT_BF16) attention_backward_bf16(a, g, st);
        else attention_backward_f32(a, g, st);
        if (parts)
            launch(distances_kernel, dim3((unsigned)((all + kWave - 1) / kWave), (unsigned)q_heads, (unsigned)shares), kWave, 0, st, a, parts, g.part_row,
                   g.first_block, g.blocks, g.q_splits, (int)share_of(z), sums);
        g.first_block += g.blocks;
    } while (!g.all_rows);
    if (const int64_t vectors = ((g.q_splits > 1 ? z.q_count() : 0) + (g.k_splits > 1 ? 2 * z.k_count() : 0)) / 4; vectors > 0) {
        const unsigned grid = (unsigned)((vectors + kAttnThreads - 1) / kAttnThreads);
        if (dt == SLIMFIT_BF16) launch(shares_kernel<uint16_t>, grid, kAttnThreads, 0, st, a, g);
        else launch(shares_kernel<float>, grid, kAttnThreads, 0, st, a, g);
    }
    if (dtable) {
        const dim3 grid((unsigned)buckets, (unsigned)q_heads);
        if (dt == SLIMFIT_BF16) launch(buckets_kernel<uint16_t>, grid, kAttnThreads, 0, st, a, sums, shares, static_cast<uint16_t *>(dtable));
        else launch(buckets_kernel<float>, grid, kAttnThreads, 0, st, a, sums, shares, static_cast<float *>(dtable));
    }
    return launch_status();
}
