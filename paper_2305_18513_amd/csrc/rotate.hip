// Attention's operands out of the rows of a QKV projection, with the norm of each query and key head and the rotation by the
// token's position on the way, the low-bit cache of what their backward pass reads, and that backward pass (not in the
// paper: decoder models' form of the reorderings in heads.hip, keys and values shared by groups of query heads).
//
//   forward   y = rot(x * rstd * gamma), rstd = (mean x^2 + eps)^-1/2; q = q_scale y, k^T = y^T, v = x
//   backward  g = rot^-1(dy), dgamma = sum g x~, dx = rstd (g gamma - x~ mean(g gamma x~)), x~ = x^ rstd
//
// A head's row is L lanes' 16-byte vectors (L a power of two), so that the row's sum is a butterfly over L lanes, the element that one
// is turned with is in the lane's own vector or in that of one other lane, and a quantisation block is block / E lanes.  A workgroup
// owns 1024 / L rows (token by token, batch by batch) in four passes, or half as many in two, and one head of the keys, or up to
// four of the queries or values one after the other, the angles of two passes' rows, times gains and factor, in registers for all of
// them.  Keys go through LDS (rows an odd number of words apart) into their transposed place.  No load or store of the head loop stands
// behind a branch: behind one, each load was waited for together with the stores before it (16384 x 48 heads of 128, bf16, 8 bits,
// forward 159 us, with them free 149, with the angles and gains in vectors 119, four heads a workgroup instead of eight 103).
//
// Bound by HBM, with 30 to 65 % on top for the start of each workgroup (place, angles and gains are asked for one after the other, of
// which only the angles have to wait for the place) and for the vector instructions (145 a 16-byte vector, half of the time) that
// do not overlap with it: that size 103 us forward (486 MB, 4.7 TB/s) and 102 backward, four heads a workgroup; 64 wide heads, two a
// workgroup, 56 and 57 (239 MB each, 38 at the stream's rate); 7289 x 36 of 64 fp32, one a workgroup, 36 and 36 (141 MB, 23);
// copies without norm and rotation 5.2 to 5.4 TB/s; a 1 : 1 stream of the card 6.2.  bf16 runs with four waves a SIMD forward
// (115 registers; five and six by spilling were slower) and three backward (162; four were not tried); angles for one pass or four
// at a time were slower.
#include "elements.hpp"

#include <type_traits>

namespace slimfit {
namespace {

constexpr int kThreads = 256;
constexpr int kPasses = 4;
constexpr int kHeld = 2;                   // passes whose angles are held at a time
constexpr int kTileWords = 4096 + 256;     // 1024 / L rows of 4 L + 1 words, L >= 4

struct Shape {
    uint32_t rows, tokens, q_heads, kv_heads, dim;         // rows = batch * tokens
    uint32_t per, q_units, units;                          // heads a query (or value) unit, units of queries, of all
    uint32_t passes, tiles;                                // of a workgroup, 2 or 4; tiles of as many rows
    uint32_t positions, half;                              // half = rotary_dim / 2; 0: no rotation
    uint32_t adjacent;
    int group, block_shift;                                // lanes of a quantisation block; log2 of its elements
    float eps, inv_dim, q_scale;
    Divide by_tokens, by_dim, by_units;
};

// Workgroups go to the eight XCDs in turn; an XCD's take consecutive units, so that what the heads of a row write side by side
// (codes, scales, rstd) becomes whole lines in its L2.
__device__ __forceinline__ uint32_t in_turn(uint32_t b, uint32_t n)
{
    const uint32_t each = n / 8;
    return b < each * 8 ? b % 8 * each + b / 8 : b;
}

// N floats, N * 4 bytes aligned
template <int N>
__device__ __forceinline__ void load_floats(const float *p, float (&f)[N])
{
    typedef float Run __attribute__((ext_vector_type(N < 4 ? N : 4)));
#pragma unroll
    for (int i = 0; i < N; i += N < 4 ? N : 4) {
        const Run r = *reinterpret_cast<const Run *>(p + i);
#pragma unroll
        for (int k = 0; k < (N < 4 ? N : 4); ++k) f[i + k] = r[k];
    }
}
// What the E elements at e0 of a row become: c x + s partner(x), without the row's rstd.  BACK: by the angle back.  False: they are not
// turned, s is 0.
template <int E, bool BACK>
__device__ __forceinline__ bool load_angles(const float *__restrict__ table, const int32_t *__restrict__ ids, const Shape &z, uint32_t row, uint32_t t,
                                            uint32_t e0, float (&c)[E], float (&s)[E])
{
#pragma unroll
    for (int i = 0; i < E; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
    const uint32_t place = ids ? (uint32_t)ids[row] : t;
    if (e0 >= 2 * z.half || place >= z.positions) return false;        // and padding
    const float *at = table + (int64_t)place * (2 * z.half);
    if (z.adjacent) {
        float a[E / 2], b[E / 2];
        load_floats<E / 2>(at + e0 / 2, a);
        load_floats<E / 2>(at + z.half + e0 / 2, b);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            c[i] = a[i / 2];
            s[i] = (i % 2 == 0) != BACK ? -b[i / 2] : b[i / 2];
        }
    } else {
        const bool low = e0 < z.half;
        at += low ? e0 : e0 - z.half;
        load_floats<E>(at, c);
        load_floats<E>(at + z.half, s);
#pragma unroll
        for (int i = 0; i < E; ++i) s[i] = low != BACK ? -s[i] : s[i];
    }
    return true;
}
// c and s times a factor and the gains of the elements and of their partners; from: the lane of those
template <int E>
__device__ __forceinline__ void weigh_angles(const float *__restrict__ gains, float factor, int from, const Shape &z, uint32_t e0, float (&c)[E], float (&s)[E])
{
    float own[E], other[E];
    load_floats<E>(gains + e0, own);
#pragma unroll
    for (int i = 0; i < E; ++i) own[i] *= factor;
    if (z.adjacent) {
#pragma unroll
        for (int i = 0; i < E; ++i) other[i] = own[i ^ 1];
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) other[i] = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(from * 4, __builtin_bit_cast(int, own[i])));
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        c[i] *= own[i];
        s[i] *= other[i];
    }
}
// c x + s partner(x) of a vector; from: the lane that holds the partners, where they are not its own neighbours.  Those of a vector that
// is not turned count as 0, whatever they are (0 times infinity would not be nothing).
template <typename T>
__device__ __forceinline__ void turn(const typename Vec<T>::raw &x, const float (&f)[Vec<T>::V], const float (&c)[Vec<T>::V], const float (&s)[Vec<T>::V],
                                     bool turned, int from, const Shape &z, float (&y)[Vec<T>::V])
{
    constexpr int E = Vec<T>::V;
    float other[E];
    if (z.adjacent) {
#pragma unroll
        for (int i = 0; i < E; ++i) other[i] = turned ? f[i ^ 1] : 0.0f;
    } else {                                               // as they lie in memory: four words
        const u32x4 mine = __builtin_bit_cast(u32x4, x);
        u32x4 theirs;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int word = (int)mine[i];
            const uint32_t got = (uint32_t)__builtin_amdgcn_ds_bpermute(from * 4, word);
            theirs[i] = turned ? got : 0u;
        }
        Vec<T>::unpack(__builtin_bit_cast(typename Vec<T>::raw, theirs), other);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = fmaf(other[i], s[i], f[i] * c[i]);
}

// A workgroup's rows of one key head between their two layouts: a thread moves E tokens of WIDE elements, 16 bytes of each (a row of
// tokens may begin anywhere: the card takes vectors at their elements' alignment), or one element at a time where a run of E
// ends past its batch, or where no row is that long.
template <typename T, bool IN, bool WHOLE>
__device__ __forceinline__ void through(uint32_t *tile, uint32_t pitch, T *kt, const Shape &z, uint32_t row0, uint32_t n_rows, uint32_t head)
{
    constexpr uint32_t E = Vec<T>::V, WIDE = 4 / sizeof(T);
    const uint32_t shift = __builtin_ctz(n_rows / E);      // (a power of two)
    typedef uint32_t Run __attribute__((ext_vector_type(4), aligned(2)));
    T *const elements = reinterpret_cast<T *>(tile);
    const uint32_t step = pitch * WIDE;
    // Rows that all begin on 16 bytes stream past the caches; of others, two workgroups share lines, which the L2 puts together
    // (37 x 12 heads x 197 x 64 fp32 forward 36.3 -> 33.0 us and backward 45 -> 39; 8 x 8 x 2048 x 128 bf16, the other way, 104 -> 108).
    auto fetch = [&](const T *at) {
        const Run *p = reinterpret_cast<const Run *>(at);
        if constexpr (WHOLE) return __builtin_nontemporal_load(p);
        else return *p;
    };
    auto put = [&](T *at, Run v) {
        Run *p = reinterpret_cast<Run *>(at);
        if constexpr (WHOLE) __builtin_nontemporal_store(v, p);
        else *p = v;
    };
    auto one = [&](T *at, uint32_t r, uint32_t d) {
        if constexpr (IN) elements[r * step + d] = *at;
        else *at = elements[r * step + d];
    };
    if (!WHOLE && z.tokens < E) {                          // along the elements, then the tokens
        for (uint32_t i = threadIdx.x; i < n_rows * z.dim; i += kThreads) {
            const uint32_t r = z.by_dim(i), d = i - r * z.dim, row = row0 + r, b = z.by_tokens(row), t = row - b * z.tokens;
            if (row < z.rows) one(kt + (((int64_t)b * z.kv_heads + head) * z.dim + d) * z.tokens + t, r, d);
        }
        return;
    }
    for (uint32_t i = threadIdx.x; i < z.dim / WIDE << shift; i += kThreads) {
        const uint32_t r = (i & ((1u << shift) - 1)) * E, d = (i >> shift) * WIDE, row = row0 + r;
        if (row >= z.rows) continue;
        const uint32_t b = z.by_tokens(row), t = row - b * z.tokens;
        T *at = kt + (((int64_t)b * z.kv_heads + head) * z.dim + d) * z.tokens + t;
        if (!WHOLE && t + E > z.tokens) {
            for (uint32_t e = 0; e < E && row + e < z.rows; ++e) {
                const uint32_t bb = z.by_tokens(row + e), tt = row + e - bb * z.tokens;
                T *to = kt + (((int64_t)bb * z.kv_heads + head) * z.dim + d) * z.tokens + tt;
                for (uint32_t k = 0; k < WIDE; ++k) one(to + (int64_t)k * z.tokens, r + e, d + k);
            }
            continue;
        }
        uint32_t *words = tile + r * pitch + d / WIDE;
        if constexpr (WIDE == 1) {
            if constexpr (IN) {
                const Run v = fetch(at);
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) words[e * pitch] = v[e];
            } else {
                Run v;
#pragma unroll
                for (uint32_t e = 0; e < E; ++e) v[e] = words[e * pitch];
                put(at, v);
            }
        } else {
            T *const next = at + z.tokens;
            if constexpr (IN) {
                const Run v = fetch(at);
                const Run u = fetch(next);
#pragma unroll
                for (uint32_t e = 0; e < E; e += 2) {
                    words[e * pitch] = __builtin_amdgcn_perm(u[e / 2], v[e / 2], 0x05040100u);
                    words[(e + 1) * pitch] = __builtin_amdgcn_perm(u[e / 2], v[e / 2], 0x07060302u);
                }
            } else {
                Run v, u;
#pragma unroll
                for (uint32_t e = 0; e < E; e += 2) {
                    const uint32_t x = words[e * pitch], y = words[(e + 1) * pitch];
                    v[e / 2] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                    u[e / 2] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                }
                put(at, v);
                put(next, u);
            }
        }
    }
}

template <typename T, bool IN>
__device__ __forceinline__ void through_tile(uint32_t *tile, T *kt, const Shape &z, uint32_t row0, uint32_t n_rows, uint32_t head)
{
    const uint32_t pitch = z.dim * sizeof(T) / 4 + 1;
    if (z.tokens % Vec<T>::V == 0) through<T, IN, true>(tile, pitch, kt, z, row0, n_rows, head);
    else through<T, IN, false>(tile, pitch, kt, z, row0, n_rows, head);
}

// the T at byte `at` (below 2^31) from a place that is the same for the workgroup
template <typename P, typename T>
__device__ __forceinline__ P *beyond(T *base, uint32_t at)
{
    using C = std::conditional_t<std::is_const_v<T>, const char, char>;
    return reinterpret_cast<P *>(reinterpret_cast<C *>(base) + at);
}

// A thread's place: rows row0 + pass * SLOTS + slot, elements e0 .. e0 + E - 1 of each head.  Lanes past a head's end do what the
// lanes L / 2 before them do (whole quantisation blocks, where there are any), rows past the last what the last does, to the same
// places: no load or store stands behind a branch, and each is waited for by itself.  counts: not such a lane.
template <typename T, int L>
struct Place {
    static constexpr int E = Vec<T>::V, SLOTS = kThreads / L;
    uint32_t unit, tiled, row0, n_rows, lane, slot, e0;
    bool counts;
    __device__ __forceinline__ Place(const Shape &z, uint32_t first)
    {
        const uint32_t at = first + in_turn(blockIdx.x, gridDim.x);
        tiled = __builtin_amdgcn_readfirstlane(z.by_units(at));
        unit = at - tiled * z.units;
        n_rows = SLOTS * z.passes;
        row0 = tiled * n_rows;
        lane = threadIdx.x % L;
        slot = threadIdx.x / L;
        const uint32_t vectors = z.dim / E;                // more than L / 2, or L is 4 and nothing is cached
        counts = lane < vectors;
        if (!counts) lane = lane >= L / 2 && lane - L / 2 < vectors ? lane - L / 2 : 0;
        e0 = lane * E;
    }
    __device__ __forceinline__ uint32_t line(const Shape &z, int pass) const    // of the tile's rows
    {
        return min(pass * SLOTS + slot, min(n_rows, z.rows - row0) - 1);
    }
    __device__ __forceinline__ bool twice(const Shape &z, int pass) const { return row0 + pass * SLOTS + slot >= z.rows; }
    // element e0 of a head of a token in a tensor (batch, heads, tokens, dim)
    __device__ __forceinline__ int64_t apart(const Shape &z, uint32_t row, uint32_t heads) const
    {
        const uint32_t batch = z.by_tokens(row), token = row - batch * z.tokens;
        return ((int64_t)batch * heads * z.tokens + token) * z.dim + e0;
    }
    __device__ __forceinline__ int partner(const Shape &z) const               // the lane of the wave that holds this one's partners
    {
        const int own = (threadIdx.x & (kWave - 1) & ~(L - 1)) + lane;
        return z.adjacent || e0 >= 2 * z.half ? own : e0 < z.half ? own + (int)(z.half / E) : own - (int)(z.half / E);
    }
};

// The values' way between the rows and (batch, head, token, element)
template <typename T, int L, bool SPLIT>
__device__ __forceinline__ void copy_values(const Place<T, L> &w, const Shape &z, T *rows, T *v)
{
    using raw = typename Vec<T>::raw;
    const uint32_t every = z.q_heads + 2 * z.kv_heads, h0 = (w.unit - z.q_units - z.kv_heads) * z.per, h1 = min(h0 + z.per, z.kv_heads);
    rows += ((int64_t)w.row0 * every + z.q_heads + z.kv_heads) * z.dim;
    uint32_t at[kPasses];
    T *to[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const uint32_t line = w.line(z, p);
        at[p] = (line * every * z.dim + w.e0) * (uint32_t)sizeof(T);
        to[p] = v + w.apart(z, w.row0 + line, z.kv_heads);
    }
    const int64_t head = (int64_t)z.tokens * z.dim;
    for (uint32_t h = h0; h < h1; ++h) {
        T *const base = rows + h * z.dim;
        raw x[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) x[p] = load_global<true>(SPLIT ? beyond<const raw>(base, at[p]) : reinterpret_cast<const raw *>(to[p] + h * head));
#pragma unroll
        for (int p = 0; p < kPasses; ++p) store_global<true>(SPLIT ? reinterpret_cast<raw *>(to[p] + h * head) : beyond<raw>(base, at[p]), x[p]);
    }
}

// MODE: no norm, a norm and no cache, or the bits of its cache
constexpr int kNoNorm = 0, kNoCache = 1;

// What a workgroup takes of the row: heads h0 .. h1 - 1 of it, and how they lie apart
struct Part {
    uint32_t h0, h1, first, heads;         // first: head of the row that is the tensor's head 0, of `heads`
    float factor;
    __device__ __forceinline__ Part(const Shape &z, uint32_t unit)
    {
        const bool key = unit >= z.q_units;
        h0 = key ? z.q_heads + unit - z.q_units : unit * z.per;
        h1 = key ? h0 + 1 : min(h0 + z.per, z.q_heads);
        first = key ? z.q_heads : 0;
        heads = key ? z.kv_heads : z.q_heads;
        factor = key ? 1.0f : z.q_scale;
    }
};

// KEY: through the tile; otherwise straight to `apart`, which is (batch, head, token, element)
template <typename T, int L, int MODE, bool KEY>
__device__ __forceinline__ void forward_heads(const Place<T, L> &w, const Part &part, const Shape &z, uint32_t *tile, const T *qkv, const float *gains,
                                              const float *table, const int32_t *ids, T *apart, float *rstd, uint8_t *codes, float *scales)
{
    using raw = typename Vec<T>::raw;
    constexpr int E = Vec<T>::V, BITS = MODE > kNoCache ? MODE : 8;
    const uint32_t every = z.q_heads + 2 * z.kv_heads, normed = z.q_heads + z.kv_heads;
    const uint32_t h0 = part.h0, h1 = part.h1;
    const int from = w.partner(z);
    const uint32_t pitch = z.dim * sizeof(T) / 4 + 1;
    const int64_t head = (int64_t)z.tokens * z.dim;
    for (int half = 0; half < (int)z.passes; half += kHeld) {
        float c[kHeld][E], s[kHeld][E];
        bool turned[kHeld];
        uint32_t line[kHeld], at[kHeld];                   // the row in the tile, the vector of its first head
        T *to[kHeld];
#pragma unroll
        for (int p = 0; p < kHeld; ++p) {
            line[p] = w.line(z, half + p);
            const uint32_t row = w.row0 + line[p];
            at[p] = (line[p] * every * z.dim + w.e0) * (uint32_t)sizeof(T);
            if constexpr (!KEY) to[p] = apart + w.apart(z, row, part.heads) - part.first * head;
            turned[p] = load_angles<E, false>(table, ids, z, row, row - z.by_tokens(row) * z.tokens, w.e0, c[p], s[p]);
            if constexpr (MODE != kNoNorm) {
                weigh_angles<E>(gains, part.factor, from, z, w.e0, c[p], s[p]);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) { c[p][i] *= part.factor; s[p][i] *= part.factor; }
            }
        }
        const T *rows = qkv + (int64_t)w.row0 * every * z.dim;
        raw x[kHeld];
        auto load = [&](uint32_t h) {
#pragma unroll
            for (int p = 0; p < kHeld; ++p) x[p] = load_global<true>(beyond<const raw>(rows + h * z.dim, at[p]));
        };
        auto take = [&](uint32_t h, auto more) {
            raw now[kHeld];
            float f[kHeld][E];
#pragma unroll
            for (int p = 0; p < kHeld; ++p) {
                now[p] = x[p];
                Vec<T>::unpack(now[p], f[p]);
            }
            if constexpr (decltype(more)::value) load(h + 1);
            if constexpr (MODE > kNoCache) {
                uint32_t a[kHeld];
#pragma unroll
                for (int p = 0; p < kHeld; ++p) {
                    float m = 0.0f;
#pragma unroll
                    for (int i = 0; i < E; ++i) m = fmaxf(m, fabsf(f[p][i]));
                    a[p] = group_max_u32(__builtin_bit_cast(uint32_t, m), z.group);
                }
                float mult[kHeld], scale;
                quad_scales<BITS, kHeld>(a, (int)threadIdx.x, mult, scale);
                static_assert(kHeld == 2, "a lane's scale is that of the pass of its lowest bit");
                const uint32_t own = threadIdx.x & 1 ? line[1] : line[0];
                *beyond<float>(scales + ((((int64_t)w.row0 * normed + h) * z.dim) >> z.block_shift), (own * normed * z.dim + w.e0) >> z.block_shift << 2) = scale;
                uint8_t *base = codes + ((int64_t)w.row0 * normed + h) * z.dim * BITS / 8;
#pragma unroll
                for (int p = 0; p < kHeld; ++p) {
                    uint32_t word[2];
                    pack_codes<BITS, E>(f[p], mult[p], word);
                    const uint32_t place = (line[p] * normed * z.dim + w.e0) * BITS / 8;
                    if (E * BITS == 16) *beyond<uint16_t>(base, place) = (uint16_t)word[0];
                    else if (E * BITS == 32) *beyond<uint32_t>(base, place) = word[0];
                    else *beyond<u32x2>(base, place) = u32x2{word[0], word[1]};
                }
            }
#pragma unroll
            for (int p = 0; p < kHeld; ++p) {
                float y[E];
                turn<T>(now[p], f[p], c[p], s[p], turned[p], from, z, y);
                if constexpr (MODE != kNoNorm) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < E; ++i) sum = fmaf(f[p][i], f[p][i], sum);
                    const float r = __builtin_amdgcn_rsqf(fmaf(group_sum_f32(w.counts ? sum : 0.0f, L), z.inv_dim, z.eps));
                    *beyond<float>(rstd + ((int64_t)w.row0 * normed + h), line[p] * normed * 4) = r;
#pragma unroll
                    for (int i = 0; i < E; ++i) y[i] *= r;
                }
                const raw out = Vec<T>::pack(y);
                if constexpr (!KEY) {
                    store_global<true>(reinterpret_cast<raw *>(to[p] + h * head), out);
                } else {
                    uint32_t *words = tile + line[p] * pitch + w.lane * 4;
                    const u32x4 held = __builtin_bit_cast(u32x4, out);
#pragma unroll
                    for (int i = 0; i < 4; ++i) words[i] = held[i];
                }
            }
        };
        load(h0);
        for (uint32_t h = h0; h + 1 < h1; ++h) take(h, std::true_type{});
        take(h1 - 1, std::false_type{});
    }
}

template <typename T, int L, int MODE>
__global__ void __launch_bounds__(kThreads)
forward_kernel(const T *__restrict__ qkv, const float *__restrict__ gamma_q, const float *__restrict__ gamma_k, const float *__restrict__ table,
               const int32_t *__restrict__ ids, T *__restrict__ q, T *__restrict__ kt, T *__restrict__ v, float *__restrict__ rstd,
               uint8_t *__restrict__ codes, float *__restrict__ scales, Shape z, uint32_t first)
{
    __shared__ uint32_t tile[kTileWords];
    const Place<T, L> w(z, first);
    if (w.unit >= z.q_units + z.kv_heads) {
        copy_values<T, L, true>(w, z, const_cast<T *>(qkv), v);
        return;
    }
    const Part part(z, w.unit);
    const bool key = w.unit >= z.q_units;
    if (!key || z.tokens == 1) {                           // (a single token's keys lie as its queries do)
        forward_heads<T, L, MODE, false>(w, part, z, tile, qkv, key ? gamma_k : gamma_q, table, ids, key ? kt : q, rstd, codes, scales);
        return;
    }
    forward_heads<T, L, MODE, true>(w, part, z, tile, qkv, gamma_k, table, ids, nullptr, rstd, codes, scales);
    __syncthreads();
    through_tile<T, false>(tile, kt, z, w.row0, w.n_rows, w.unit - z.q_units);
}

// sums: of g x~, over the thread's rows
template <typename T, int L, int MODE, bool KEY>
__device__ __forceinline__ void backward_heads(const Place<T, L> &w, const Part &part, const Shape &z, const uint32_t *tile, const T *apart, const T *qkv, const uint8_t *codes,
                                               const float *scales, const float *rstd, const float *gains, const float *table, const int32_t *ids, T *dqkv,
                                               float (&sums)[Vec<T>::V])
{
    using raw = typename Vec<T>::raw;
    constexpr int E = Vec<T>::V, BITS = MODE > kNoCache ? MODE : 8;
    const uint32_t every = z.q_heads + 2 * z.kv_heads, normed = z.q_heads + z.kv_heads;
    const uint32_t h0 = part.h0, h1 = part.h1;
    const int from = w.partner(z);
    const uint32_t pitch = z.dim * sizeof(T) / 4 + 1;
    const int64_t head = (int64_t)z.tokens * z.dim;
    float gamma[MODE == kNoNorm ? 1 : E];
    if constexpr (MODE != kNoNorm) {
#pragma unroll
        for (int i = 0; i < E; ++i) gamma[i] = gains[w.e0 + i];
    }
    for (int half = 0; half < (int)z.passes; half += kHeld) {
        float c[kHeld][E], s[kHeld][E], counts[kHeld];
        bool turned[kHeld];
        uint32_t line[kHeld];
        const T *at[kHeld];
#pragma unroll
        for (int p = 0; p < kHeld; ++p) {
            line[p] = w.line(z, half + p);
            counts[p] = w.twice(z, half + p) ? 0.0f : 1.0f;
            const uint32_t row = w.row0 + line[p];
            if constexpr (!KEY) at[p] = apart + w.apart(z, row, part.heads) - part.first * head;
            turned[p] = load_angles<E, true>(table, ids, z, row, row - z.by_tokens(row) * z.tokens, w.e0, c[p], s[p]);
#pragma unroll
            for (int i = 0; i < E; ++i) { c[p][i] *= part.factor; s[p][i] *= part.factor; }
        }
        raw grad[kHeld], x[kHeld];
        uint32_t word[kHeld][2];
        float step[kHeld], r[kHeld];
        auto load = [&](uint32_t h) {
#pragma unroll
            for (int p = 0; p < kHeld; ++p) {
                if constexpr (KEY) {
                    const uint32_t *words = tile + line[p] * pitch + w.lane * 4;
                    grad[p] = __builtin_bit_cast(raw, u32x4{words[0], words[1], words[2], words[3]});
                } else {
                    grad[p] = load_global<true>(reinterpret_cast<const raw *>(at[p] + h * head));
                }
                if constexpr (MODE == kNoCache) {
                    x[p] = load_global<true>(beyond<const raw>(qkv + ((int64_t)w.row0 * every + h) * z.dim, (line[p] * every * z.dim + w.e0) * (uint32_t)sizeof(T)));
                } else if constexpr (MODE > kNoCache) {
                    const uint8_t *base = codes + ((int64_t)w.row0 * normed + h) * z.dim * BITS / 8;
                    const uint32_t place = line[p] * normed * z.dim + w.e0;
                    word[p][1] = 0u;
                    if (E * BITS == 16) word[p][0] = *beyond<const uint16_t>(base, place * BITS / 8);
                    else if (E * BITS == 32) word[p][0] = *beyond<const uint32_t>(base, place * BITS / 8);
                    else {
                        const u32x2 t = *beyond<const u32x2>(base, place * BITS / 8);
                        word[p][0] = t.x;
                        word[p][1] = t.y;
                    }
                    step[p] = *beyond<const float>(scales + ((((int64_t)w.row0 * normed + h) * z.dim) >> z.block_shift), place >> z.block_shift << 2);
                }
                if constexpr (MODE != kNoNorm) r[p] = *beyond<const float>(rstd + ((int64_t)w.row0 * normed + h), line[p] * normed * 4);
            }
        };
        auto take = [&](uint32_t h, auto more) {
            T *const rows = dqkv + ((int64_t)w.row0 * every + h) * z.dim;
            float g[kHeld][E], xn[kHeld][E], root[kHeld];
#pragma unroll
            for (int p = 0; p < kHeld; ++p) {
                float f[E];
                Vec<T>::unpack(grad[p], f);
                turn<T>(grad[p], f, c[p], s[p], turned[p], from, z, g[p]);
                if constexpr (MODE == kNoCache) {
                    root[p] = r[p];
                    Vec<T>::unpack(x[p], xn[p]);
#pragma unroll
                    for (int i = 0; i < E; ++i) xn[p][i] *= root[p];
                } else if constexpr (MODE > kNoCache) {
                    root[p] = r[p];
                    const float by = step[p] * root[p];
#pragma unroll
                    for (int i = 0; i < E; ++i) xn[p][i] = (float)code_field<BITS>(word[p][i * BITS / 32], i % (32 / BITS)) * by;
                }
            }
            if constexpr (decltype(more)::value) load(h + 1);
#pragma unroll
            for (int p = 0; p < kHeld; ++p) {
                if constexpr (MODE != kNoNorm) {
                    float dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        sums[i] = fmaf(g[p][i] * counts[p], xn[p][i], sums[i]);
                        g[p][i] *= gamma[i];
                        dot = fmaf(g[p][i], xn[p][i], dot);
                    }
                    dot = group_sum_f32(w.counts ? dot : 0.0f, L) * z.inv_dim;
#pragma unroll
                    for (int i = 0; i < E; ++i) g[p][i] = root[p] * fmaf(-xn[p][i], dot, g[p][i]);
                }
                store_global<true>(beyond<raw>(rows, (line[p] * every * z.dim + w.e0) * (uint32_t)sizeof(T)), Vec<T>::pack(g[p]));
            }
        };
        load(h0);
        for (uint32_t h = h0; h + 1 < h1; ++h) take(h, std::true_type{});
        take(h1 - 1, std::false_type{});
    }
}

// partial: [units of queries, units of keys] x row tiles x dim sums of a workgroup each, or null where they are not asked for
template <typename T, int L, int MODE>
__global__ void __launch_bounds__(kThreads)
backward_kernel(const T *__restrict__ dq, const T *__restrict__ dkt, const T *__restrict__ dv, const T *__restrict__ qkv, const uint8_t *__restrict__ codes,
                const float *__restrict__ scales, const float *__restrict__ rstd, const float *__restrict__ gamma_q, const float *__restrict__ gamma_k,
                const float *__restrict__ table, const int32_t *__restrict__ ids, T *__restrict__ dqkv, float *__restrict__ partial, Shape z, uint32_t first)
{
    constexpr int E = Vec<T>::V, SLOTS = kThreads / L;
    __shared__ uint32_t tile[kTileWords];
    const Place<T, L> w(z, first);
    float sums[E];
#pragma unroll
    for (int i = 0; i < E; ++i) sums[i] = 0.0f;
    if (w.unit >= z.q_units + z.kv_heads) {
        copy_values<T, L, false>(w, z, dqkv, const_cast<T *>(dv));
        return;
    }
    const Part part(z, w.unit);
    const bool key = w.unit >= z.q_units;
    if (!key || z.tokens == 1) {
        backward_heads<T, L, MODE, false>(w, part, z, tile, key ? dkt : dq, qkv, codes, scales, rstd, key ? gamma_k : gamma_q, table, ids, dqkv, sums);
    } else {
        through_tile<T, true>(tile, const_cast<T *>(dkt), z, w.row0, w.n_rows, w.unit - z.q_units);
        __syncthreads();
        backward_heads<T, L, MODE, true>(w, part, z, tile, nullptr, qkv, codes, scales, rstd, gamma_k, table, ids, dqkv, sums);
    }
    if constexpr (MODE != kNoNorm) {
        if (!partial) return;                              // (uniform for the launch)
        __syncthreads();                                   // the tile is read
        float *rows = reinterpret_cast<float *>(tile);     // SLOTS x dim
        if (w.counts) {
#pragma unroll
            for (int i = 0; i < E; ++i) rows[w.slot * z.dim + w.e0 + i] = sums[i];
        }
        __syncthreads();
        float *to = partial + ((int64_t)w.unit * z.tiles + w.tiled) * z.dim;
        for (uint32_t d = threadIdx.x; d < z.dim; d += kThreads) {
            float total = 0.0f;
            for (int k = 0; k < SLOTS; ++k) total += rows[k * z.dim + d];
            to[d] = total;
        }
    }
}

// dgamma[d] = sum over the partial sums of its side.  A workgroup: 16 columns, 64 slices of the rows.
constexpr int kGammaThreads = 1024;
__global__ void __launch_bounds__(kGammaThreads)
gamma_kernel(const float *__restrict__ partial, uint32_t dim, int64_t q_rows, int64_t k_rows, float *__restrict__ dgamma_q, float *__restrict__ dgamma_k)
{
    constexpr int SLICES = kGammaThreads / 16;
    __shared__ double sums[kGammaThreads];
    const uint32_t blocks = gridDim.x / 2, side = blockIdx.x / blocks, d = blockIdx.x % blocks * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
    const float *from = partial + (side ? q_rows * dim : 0);
    const int64_t n = side ? k_rows : q_rows;
    double total = 0.0;
    if (d < dim) {
#pragma unroll 8
        for (int64_t i = slice; i < n; i += SLICES) total += (double)from[i * dim + d];
    }
    sums[threadIdx.x] = total;
    __syncthreads();
    if (slice < 4) {
#pragma unroll
        for (int k = 4; k < SLICES; k += 4) total += sums[k * 16 + threadIdx.x];
        sums[threadIdx.x] = total;
    }
    __syncthreads();
    if (slice == 0 && d < dim) (side ? dgamma_k : dgamma_q)[d] = (float)((sums[threadIdx.x] + sums[threadIdx.x + 16]) + (sums[threadIdx.x + 32] + sums[threadIdx.x + 48]));
}

int lanes_of(int32_t dt, int32_t dim)
{
    const int vectors = dim / (dt == SLIMFIT_F32 ? 4 : 8);
    int L = 4;
    while (L < vectors) L *= 2;
    return L;
}

// Heads a query (or value) workgroup takes one after the other: as many as leave four workgroups to a compute unit, at most 4.
// (Forward and backward in us with one, two and four: 16 384 x 48 heads of 128 bf16 251, 214, 213; 16 384 x 48 of 64, which take
// two, 121, 112, 121, and at 16 000 tokens, where it is one, 119, 111, 119; 7296 x 36 of 64 fp32, one, 70, 70, 73.)
int heads_each(int64_t tiles, int32_t heads)
{
    int per = 4;
    while (per > 1 && tiles * ((heads + per - 1) / per) < 1024) per /= 2;
    return per;
}

int32_t validate(int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim)
{
    if (!dtype_ok(dt) || batch < 0 || tokens < 0 || q_heads < 1 || kv_heads < 1 || dim < 1 || q_heads % kv_heads != 0) return SLIMFIT_ERR_INVALID_ARG;
    if (dim % (dt == SLIMFIT_F32 ? 4 : 8) != 0 || dim > 256) return SLIMFIT_ERR_UNSUPPORTED;
    if (batch == 0 || tokens == 0) return SLIMFIT_OK;
    if (batch >= ((int64_t)1 << 31) / tokens || ((int64_t)q_heads + 2 * (int64_t)kv_heads) * dim > (1 << 20)) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

// A workgroup takes four passes, or two where that would be fewer workgroups than this.  (Forward and backward in us with two and four,
// and the workgroups of four: 48 heads of 64 bf16 with 8 bits, 16 384 tokens 120 and 112, 4096, though 13 312 tokens 98 and 101,
// 4992; 48 of 128, 8192 tokens 109 and 115, 2304, 12 288 tokens 157 and 158, 3456; 40 of 96, nothing kept, 4096 tokens 47 and 54,
// 2560, though 6144 tokens 66 and 64, 2304.  Forward alone a prompt of 4097 x 40 of 96 19.0 and 23.5, 2600, 512 x 48 of 64 7.3 and
// 7.9, 192.)
constexpr int64_t kBusy = 4000;

struct Plan {
    int L, per, passes;
    int64_t tiles, q_units, v_units, blocks;
    Plan(int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim)
    {
        L = lanes_of(dt, dim);
        for (passes = 4;; passes = 2) {
            const int64_t each = 256 * passes / L;
            tiles = (batch * tokens + each - 1) / each;
            per = heads_each(tiles, q_heads);
            q_units = (q_heads + per - 1) / per;
            v_units = (kv_heads + per - 1) / per;
            blocks = tiles * (q_units + kv_heads + v_units);
            if (passes == 2 || blocks >= kBusy) break;
        }
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

Shape shape_of(const Plan &p, const Rotation &r, int32_t dt, int64_t batch, int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t dim, float eps, float q_scale, int32_t bits,
               int32_t block)
{
    const uint32_t units = (uint32_t)(p.q_units + kv_heads + p.v_units);
    Shape z = {(uint32_t)(batch * tokens), (uint32_t)tokens, (uint32_t)q_heads, (uint32_t)kv_heads, (uint32_t)dim, (uint32_t)p.per, (uint32_t)p.q_units,
               units, (uint32_t)p.passes, (uint32_t)p.tiles, (uint32_t)r.positions, (uint32_t)r.rotary_dim / 2, r.rotary_dim > 0 && r.pairing == SLIMFIT_ROTARY_ADJACENT, 4, 0, eps, 1.0f / (float)dim, q_scale,
               Divide((uint32_t)tokens), Divide((uint32_t)dim), Divide(units)};
    if (bits != 0) {
        z.group = block / (dt == SLIMFIT_F32 ? 4 : 8);
        z.block_shift = __builtin_ctz((unsigned)block);
    }
    return z;
}

// f(T{}, L, MODE) for the call's type, lanes a head and mode
template <typename F>
void choose(int32_t dt, int L, bool norm, int32_t bits, F f)
{
    auto with_bits = [&](auto t, auto l) {
        if (!norm) f(t, l, std::integral_constant<int, kNoNorm>{});
        else if (bits == 0) f(t, l, std::integral_constant<int, kNoCache>{});
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
    const Shape z = shape_of(plan, turn, dt, batch, tokens, q_heads, kv_heads, head_dim, eps, q_scale, bits, block);
    hipStream_t st = static_cast<hipStream_t>(stream);
    constexpr int64_t kMost = kMaxGridThreads / kThreads;
    for (int64_t first = 0; first < plan.blocks; first += kMost) {
        const unsigned here = (unsigned)(plan.blocks - first < kMost ? plan.blocks - first : kMost);
        choose(dt, plan.L, norm, bits, [&](auto t, auto l, auto b) {
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
        launch(gamma_kernel, gamma_blocks, kGammaThreads, 0, st, nullptr, (uint32_t)head_dim, 0, 0, dgamma_q, dgamma_k);      // sums of nothing
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
    const Shape z = shape_of(plan, turn, dt, batch, tokens, q_heads, kv_heads, head_dim, 0.0f, q_scale, bits, block);
    float *partial = want ? static_cast<float *>(workspace) : nullptr;
    constexpr int64_t kMost = kMaxGridThreads / kThreads;
    for (int64_t first = 0; first < plan.blocks; first += kMost) {
        const unsigned here = (unsigned)(plan.blocks - first < kMost ? plan.blocks - first : kMost);
        choose(dt, plan.L, norm, bits, [&](auto t, auto l, auto b) {
            using T = decltype(t);
            launch(backward_kernel<T, decltype(l)::value, decltype(b)::value>, here, kThreads, 0, st, static_cast<const T *>(dq),
                   static_cast<const T *>(dkt), static_cast<const T *>(dv), static_cast<const T *>(qkv), codes, scales, rstd, gamma_q, gamma_k, table,
                   position_ids, static_cast<T *>(dqkv), partial, z, (uint32_t)first);
        });
    }
    if (want)
        launch(gamma_kernel, gamma_blocks, kGammaThreads, 0, st, partial, (uint32_t)head_dim, plan.tiles * plan.q_units, plan.tiles * (int64_t)kv_heads, dgamma_q,
               dgamma_k);
    return launch_status();
}
