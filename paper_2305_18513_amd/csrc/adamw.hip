// AdamW over all tensors of a model in one launch, with Eq. 1's distance of each layer from the same pass:
//     g' = factor g,   m' = b1 m + (1 - b1) g',   v' = b2 v + ((1 - b2) g') g',
//     d = -(lr decay w + lr / (1 - b1^t) * m' / (sqrt(v') / sqrt(1 - b2^t) + eps)),   w' = w + d,   distance = mean |d| / max(|w|, floor).
//
// As for the distances alone (layer_delta.hip) the tensors are cut into chunks of kChunk elements (kShort where there are few), a workgroup each, the table of
// the tensors lies in the workspace, and each workgroup's sum of terms goes out in fp64 for a second launch that adds them in order.
//
// States in 8 bits, a scale for each run of `block` elements:
//   m   e4m3 of m' * 448 / max|m'| (round to nearest even, the conversion instruction's), scale max|m'| / 448.
//   v   5 exponent and 3 fraction bits over a power of two, 2^-31 to 1 of the run's largest exponent: code c > 0 stands for
//       2^(c >> 3) (1 + (c & 7) / 8) times the scale, which is the fp32 number whose bits are the scale's + (c << 20); 0 is 0.
//       Rounding to the nearest would never let a v decay (a step takes 0.001 of it, half a step of the code is 0.06), so v' is
//       rounded up with the probability of what is cut off: 20 bits of dither are added to the fp32 bits before the cut.  The
//       dither is a function of seed, step, tensor and place alone.  A v' that is not 0 never becomes 0 (m' / eps would explode).
//       A run with a v' that is not finite is NaN as a whole, as its m is: no scale has codes for that one and for the others.
// m' and v' are rounded products and their rounded sum, without a fused multiply-add, so that the codes are defined.
//
// What bounds it: memory (fp32 weights and states, 16.8 million, 470 MB: 86 us, 5.5 TB/s; 151 million bf16 weights with states in 8 bits, 1.46 GB: 260 to
// 275 us, 5.5 TB/s, where vector instructions are as much); a small model, the launches.
#include "common.hpp"

#include <algorithm>
#include <memory>
#include <new>
#include <type_traits>

namespace slimfit {
namespace {

constexpr int kThreads = 256;
// Both multiples of every block and of a workgroup's pass.  kShort where there are up to kFew chunks otherwise, two for each compute
// unit (us with kChunk, kShort: 30 tensors of 16 384 elements 12.2, 7.7; 16 of 262 144 31.2, 22.6; 32 of those 43.8, 44.8).
constexpr int kChunk = 32 * kThreads, kShort = 8 * kThreads, kFew = 512;
// Elements of a thread at a time: with states in 32 bits 16 bytes of each, so that what a wave asks for at once is whole lines (85 million weights,
// a third frozen, in fp32: 287 us, 328 with eight elements in two vectors); with states in 8 bits 8 bytes of codes, for the work on a run's scale is
// a thread's (6 % more with four).
template <int BITS> constexpr int kPer = BITS == 8 ? 8 : 4;
constexpr int kNoNumber = 244;               // of a v over a scale of 2^98: 0x70800000 + (244 << 20) is 0x7FC00000
constexpr uint32_t kMagic = 0x534C4157u;     // "SLAW"
constexpr int kPlanBatch = 32;

struct Header {                              // 64 bytes at the start of the workspace
    uint32_t magic;
    int32_t n_layers;
    int64_t total_chunks;
    int32_t w_dt, grad_dt, bits, block, of, pad[7];         // of: elements of a chunk
};
static_assert(sizeof(Header) == 64, "header size");

struct Entry {                               // 80 bytes
    void *w;
    const void *grad;                        // NULL: frozen
    void *m, *v;
    float *m_scales, *v_scales;
    uint16_t *copy;                          // bf16 copy of fp32 weights, or NULL
    int64_t numel, first_chunk;
    float decay;
    uint32_t pad;
};
static_assert(sizeof(Entry) == 80, "entry size");

struct PlanBatch {
    Entry e[kPlanBatch];
};

inline size_t table_bytes(int32_t L) { return (sizeof(Header) + sizeof(Entry) * (size_t)L + 255) & ~(size_t)255; }

__global__ void plan_kernel(char *ws, Header h, int first, int count, PlanBatch batch)
{
    Entry *table = reinterpret_cast<Entry *>(ws + sizeof(Header));
    const int t = threadIdx.x;
    if (t < count) table[first + t] = batch.e[t];
    if (first == 0 && t == 0) *reinterpret_cast<Header *>(ws) = h;
}

struct Step {
    double beta1, beta2;
    float b1, one_b1, b2, one_b2, eps, lr, rate, root, factor, floor;
    uint32_t seed, step;
};

__host__ __device__ inline uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x6A09E667u;                        // the fraction bits of sqrt 2 and sqrt 3
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}

__host__ __device__ inline double power(double b, uint32_t n)
{
    double p = 1.0;
    for (; n; n >>= 1, b *= b)
        if (n & 1u) p *= b;
    return p;
}

template <int N> __device__ __forceinline__ void load_all(const float *p, float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const f32x4 r = load_global<true>(reinterpret_cast<const f32x4 *>(p) + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[4 * i + j] = r[j];
    }
}
template <int N> __device__ __forceinline__ void load_all(const uint16_t *p, float (&f)[N])
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 2)));
    const V r = load_global<true>(reinterpret_cast<const V *>(p));
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const uint32_t u = r[i];
        f[2 * i] = __builtin_bit_cast(float, u << 16);
        f[2 * i + 1] = __builtin_bit_cast(float, u & 0xFFFF0000u);
    }
}
template <int N> __device__ __forceinline__ void store_all(float *p, const float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) store_global<true>(reinterpret_cast<f32x4 *>(p) + i, f32x4{f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]});
}
template <int N> __device__ __forceinline__ void store_all(uint16_t *p, const float (&f)[N])
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 2)));
    V r;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) r[i] = bf16_narrow2(f[2 * i], f[2 * i + 1]);
    store_global<true>(reinterpret_cast<V *>(p), r);
}
__device__ __forceinline__ float load1(const float *p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t *p) { return bf16_widen(*p); }
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t *p, float v) { *p = (uint16_t)bf16_narrow(v); }
// n of the elements (the last vector of a tensor may have fewer), 0 in place of the others
template <typename T, int N> __device__ __forceinline__ void load_some(const T *p, int n, float (&f)[N])
{
    if (n >= N) return load_all<N>(p, f);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = j < n ? load1(p + j) : 0.0f;
}
template <typename T, int N> __device__ __forceinline__ void store_some(T *p, int n, const float (&f)[N])
{
    if (n >= N) return store_all<N>(p, f);
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) store1(p + j, f[j]);
}
template <int N> struct Codes {                             // of N elements, a byte each
    uint32_t w[N / 4];
};
template <int N> __device__ __forceinline__ Codes<N> load_codes(const uint8_t *p, int n)
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 4)));
    Codes<N> c = {};
    if (n >= N) {
        if constexpr (N == 4) {
            c.w[0] = load_global<true>(reinterpret_cast<const uint32_t *>(p));
        } else {
            const V r = load_global<true>(reinterpret_cast<const V *>(p));
#pragma unroll
            for (int i = 0; i < N / 4; ++i) c.w[i] = r[i];
        }
        return c;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) c.w[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
    return c;
}
template <int N> __device__ __forceinline__ void store_codes(uint8_t *p, int n, const Codes<N> &c)
{
    typedef uint32_t V __attribute__((ext_vector_type(N / 4)));
    if (n >= N) {
        if constexpr (N == 4) {
            store_global<true>(reinterpret_cast<uint32_t *>(p), c.w[0]);
        } else {
            V r;
#pragma unroll
            for (int i = 0; i < N / 4; ++i) r[i] = c.w[i];
            store_global<true>(reinterpret_cast<V *>(p), r);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        if (j < n) p[j] = (uint8_t)(c.w[j / 4] >> (8 * (j % 4)));
}

template <int N> __device__ __forceinline__ void decode_m(const Codes<N> &c, float scale, float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[i], true);
        f[4 * i] = a[0] * scale;
        f[4 * i + 1] = a[1] * scale;
        f[4 * i + 2] = b[0] * scale;
        f[4 * i + 3] = b[1] * scale;
    }
}
template <int N> __device__ __forceinline__ void decode_v(const Codes<N> &c, float scale, float (&f)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const uint32_t code = (c.w[j / 4] >> (8 * (j % 4))) & 255u;
        f[j] = code ? __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, scale) + (code << 20)) : 0.0f;
    }
}
// m' of a run's lanes: codes, and the scale in every lane
template <int N> __device__ __forceinline__ Codes<N> encode_m(const float (&m)[N], int lanes, float &scale)
{
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < N; ++j) top = max(top, __builtin_bit_cast(uint32_t, m[j]) & 0x7FFFFFFFu);
    const float a = __builtin_bit_cast(float, group_max_u32(top, lanes));
    const float up = 448.0f / a;
    const bool fine = !__builtin_isinf(up);                 // not a run of zeros, nor one whose factor overflows
    const float by = fine ? up : 0.0f;
    scale = fine ? a / 448.0f : 0.0f;
    Codes<N> c;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(m[4 * i] * by, m[4 * i + 1] * by, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(m[4 * i + 2] * by, m[4 * i + 3] * by, w, true);
        c.w[i] = (uint32_t)w;
    }
    return c;
}
// v' likewise; `first`: the key of the tensor's dither plus the number of the fours before these elements
template <int N> __device__ __forceinline__ Codes<N> encode_v(const float (&v)[N], int lanes, uint32_t first, float &scale)
{
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < N; ++j) top = max(top, __builtin_bit_cast(uint32_t, v[j]));
    top = group_max_u32(top, lanes) >> 23;
    const bool none = top >= 255u;                          // one is not finite: NaN, by a code that is one over this scale
    const int zero = none ? kNoNumber : 0, least = none ? kNoNumber : 1, most = none ? kNoNumber : 255;
    top = none ? 225u : top > 31u ? top - 30u : 1u;
    scale = __builtin_bit_cast(float, top << 23);
    Codes<N> c = {};
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint32_t word = mix(first + (uint32_t)i);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, v[4 * i + j]);
            const uint32_t dither = (j == 0 ? word : __builtin_rotateleft32(word, 8 * j)) >> 12;
            const int code = (int)((bits + dither) >> 20) - (int)(8u * top);
            c.w[i] |= (uint32_t)(bits ? min(max(code, least), most) : zero) << (8 * j);
        }
    }
    return c;
}

template <typename TW, typename TG, int BITS, bool SCORE>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const char *__restrict__ ws, int32_t L, int64_t total_chunks, int32_t of, int32_t block, Step s,
                                                         const float *__restrict__ live, const uint8_t *__restrict__ frozen, double *__restrict__ partials)
{
    constexpr int N = kPer<BITS>, kPass = kThreads * N;
    __shared__ double lds[kThreads / kWave];
    const Header *h = reinterpret_cast<const Header *>(ws);
    if (h->magic != kMagic || h->n_layers != L || h->total_chunks != total_chunks || h->of != of || h->bits != BITS || h->block != block ||
        h->w_dt != (sizeof(TW) == 2 ? SLIMFIT_BF16 : SLIMFIT_F32) || h->grad_dt != (sizeof(TG) == 2 ? SLIMFIT_BF16 : SLIMFIT_F32))
        return;                                             // no matching plan: touch nothing
    const Entry *table = reinterpret_cast<const Entry *>(ws + sizeof(Header));
    const int64_t chunk = blockIdx.x;
    // the last tensor whose first_chunk <= chunk: 64 of them looked at a time (a small model's step 11.1 us with one at a time, 9.9 so)
    int lo = 0;
    for (int count = L; count > 1;) {
        const int apart = (count + kWave - 1) / kWave, mine = (int)(threadIdx.x & 63) * apart;
        const uint64_t before = __builtin_amdgcn_ballot_w64(mine < count && table[lo + min(mine, count - 1)].first_chunk <= chunk);
        const int last = (__builtin_popcountll(before) - 1) * apart;
        lo += last;
        count = min(apart, count - last);
    }
    const Entry e = table[lo];
    if (!e.grad || (frozen && frozen[lo])) {
        if (SCORE && threadIdx.x == 0) partials[chunk] = 0.0;
        return;
    }
    if (live) {
        s.lr = live[0];
        s.step = (uint32_t)live[1];
        s.factor = live[2];
        s.rate = (float)((double)s.lr / (1.0 - power(s.beta1, s.step)));
        s.root = (float)(1.0 / __builtin_sqrt(1.0 - power(s.beta2, s.step)));
    }
    const int64_t off = (chunk - e.first_chunk) * of;
    const int len = (int)min((int64_t)of, e.numel - off);
    const int lanes = block / N;
    const float decay = s.lr * e.decay;
    const uint32_t key = BITS == 8 ? mix(s.seed ^ mix(s.step ^ mix((uint32_t)lo + 1u))) + (uint32_t)(off >> 2) : 0u;
    double acc = 0.0;
    auto pass = [&](auto whole, int p) {                    // (all threads together: lanes of a run stay together)
        const int at = p + threadIdx.x * N;
        const int n = decltype(whole)::value ? N : min(len - at, N);
        TW *const wp = static_cast<TW *>(e.w) + off + at;
        float w[N], g[N], m[N], v[N];
        load_some(wp, n, w);
        load_some(static_cast<const TG *>(e.grad) + off + at, n, g);
        const int64_t run = (off + at) / (BITS == 8 ? block : 1);
        if constexpr (BITS == 32) {
            load_some(static_cast<float *>(e.m) + off + at, n, m);
            load_some(static_cast<float *>(e.v) + off + at, n, v);
        } else {
            const Codes<N> cm = load_codes<N>(static_cast<uint8_t *>(e.m) + off + at, n), cv = load_codes<N>(static_cast<uint8_t *>(e.v) + off + at, n);
            decode_m(cm, n > 0 ? e.m_scales[run] : 0.0f, m);
            decode_v(cv, n > 0 ? e.v_scales[run] : 0.0f, v);
        }
        float to[N], d[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float gj = g[j] * s.factor;
            m[j] = m[j] * s.b1 + gj * s.one_b1;
            v[j] = v[j] * s.b2 + (gj * s.one_b2) * gj;
        }
        // The instructions for roots and reciprocals are within a step of the last place, and take numbers below the normal ones as 0: a root
        // of those, up to 2^-63, counts `root` times, so from an eps of 2^-40 of these on it is none of their sum.  (Divided and rooted by the
        // correctly rounded sequences, distances too and added up in fp64 one by one: 97 vector instructions an element with 8 bits instead of 59,
        // 361 us instead of 290 for 151 million bf16 weights.)
        if (s.eps >= 0x1p-40f * s.root) {
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = m[j] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[j]) * s.root + s.eps);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) d[j] = m[j] / (__builtin_sqrtf(v[j]) * s.root + s.eps);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            d[j] = -(w[j] * decay + d[j] * s.rate);
            to[j] = w[j] + d[j];
        }
        if constexpr (SCORE) {                              // (past the end d is 0)
            float q[N], least = __builtin_inff();
#pragma unroll
            for (int j = 0; j < N; ++j) {
                q[j] = fmaxf(__builtin_fabsf(w[j]), s.floor);
                least = fminf(least, q[j]);
            }
            if (least >= 0x1p-126f) {
#pragma unroll
                for (int j = 0; j < N; ++j) q[j] = __builtin_fabsf(d[j]) * __builtin_amdgcn_rcpf(q[j]);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) q[j] = d[j] != 0.0f ? __builtin_fabsf(d[j]) / q[j] : 0.0f;
            }
#pragma unroll
            for (int j = 1; j < N; j *= 2)
#pragma unroll
                for (int i = 0; i + j < N; i += 2 * j) q[i] += q[i + j];
            acc += (double)q[0];
        }
        store_some(wp, n, to);
        if (sizeof(TW) == 4 && e.copy) store_some(e.copy + off + at, n, to);
        if constexpr (BITS == 32) {
            store_some(static_cast<float *>(e.m) + off + at, n, m);
            store_some(static_cast<float *>(e.v) + off + at, n, v);
        } else {
            if (n < N) {                                 // past the end: nothing that a run's largest could be
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (j >= n) m[j] = v[j] = 0.0f;
            }
            float ms, vs;
            const Codes<N> cm = encode_m(m, lanes, ms), cv = encode_v(v, lanes, key + (uint32_t)(at >> 2), vs);
            store_codes(static_cast<uint8_t *>(e.m) + off + at, n, cm);
            store_codes(static_cast<uint8_t *>(e.v) + off + at, n, cv);
            if (n > 0 && (threadIdx.x & (lanes - 1)) == 0) {
                e.m_scales[run] = ms;
                e.v_scales[run] = vs;
            }
        }
    };
    // A pass that is whole asks for everything before it waits for anything (151 million bf16 weights, 8 bits: 290 us with a branch and a wait
    // at each load, as in a tensor's last pass, 260 so).
    for (int p = 0; p < len; p += kPass) {
        if (p + kPass <= len) pass(std::true_type(), p);
        else pass(std::false_type(), p);
    }
    if constexpr (SCORE) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) acc += __shfl_xor(acc, o, kWave);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = acc;
        __syncthreads();
        if (threadIdx.x == 0) partials[chunk] = ((lds[0] + lds[1]) + lds[2]) + lds[3];
    }
}

__global__ __launch_bounds__(kThreads) void finish_kernel(const char *__restrict__ ws, int32_t L, int64_t total_chunks, Header want,
                                                       const double *__restrict__ partials, float *__restrict__ d_out)
{
    __shared__ double lds[kThreads / kWave];
    const int layer = blockIdx.x;
    const Header *h = reinterpret_cast<const Header *>(ws);
    if (h->magic != kMagic || h->n_layers != L || h->total_chunks != total_chunks || h->of != want.of || h->bits != want.bits || h->block != want.block ||
        h->w_dt != want.w_dt || h->grad_dt != want.grad_dt) {
        if (threadIdx.x == 0) d_out[layer] = __builtin_nanf("");
        return;
    }
    const Entry &e = reinterpret_cast<const Entry *>(ws + sizeof(Header))[layer];
    const int64_t chunks = (e.numel + want.of - 1) / want.of;
    double acc = 0.0;
    for (int64_t c = threadIdx.x; c < chunks; c += kThreads) acc += partials[e.first_chunk + c];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) acc += __shfl_xor(acc, o, kWave);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = acc;
    __syncthreads();
    acc = ((lds[0] + lds[1]) + lds[2]) + lds[3];
    if (threadIdx.x == 0) d_out[layer] = e.numel > 0 ? (float)(acc / (double)e.numel) : 0.0f;
}

constexpr int kStates = 4;                   // elements of a thread that reads states back (151 million: 237 us, with eight, whose fp32 numbers are two vectors, 445)

__global__ __launch_bounds__(kThreads) void states_kernel(const uint8_t *__restrict__ m, const float *__restrict__ m_scales, const uint8_t *__restrict__ v,
                                                          const float *__restrict__ v_scales, int64_t n, int shift, float *__restrict__ m_out,
                                                          float *__restrict__ v_out, int64_t first)
{
    const int64_t at = first + ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kStates;
    if (at >= n) return;
    const int some = (int)min((int64_t)kStates, n - at);
    float a[kStates], b[kStates];
    decode_m(load_codes<kStates>(m + at, some), m_scales[at >> shift], a);
    decode_v(load_codes<kStates>(v + at, some), v_scales[at >> shift], b);
    store_some(m_out + at, some, a);
    store_some(v_out + at, some, b);
}

struct Layout {
    int64_t chunks = 0;
    int32_t of = kChunk;
    size_t bytes = 0;
};

int32_t layout_of(int32_t L, const int64_t *numel, Layout *out)
{
    if (L < 0 || (L > 0 && !numel)) return SLIMFIT_ERR_INVALID_ARG;
    int64_t chunks = 0;
    for (int32_t i = 0; i < L; ++i) {
        if (numel[i] < 0) return SLIMFIT_ERR_INVALID_ARG;
        if (numel[i] > ((int64_t)1 << 33)) return SLIMFIT_ERR_UNSUPPORTED;       // the dither counts fours of elements in 32 bits
        chunks += (numel[i] + kChunk - 1) / kChunk;
    }
    if (!grid_fits(chunks, kThreads)) return SLIMFIT_ERR_UNSUPPORTED;
    if (chunks <= kFew) {
        out->of = kShort;
        chunks = 0;
        for (int32_t i = 0; i < L; ++i) chunks += (numel[i] + kShort - 1) / kShort;
    }
    out->chunks = chunks;
    out->bytes = table_bytes(L) + sizeof(double) * (size_t)chunks;
    return SLIMFIT_OK;
}

int32_t check_kind(int32_t w_dt, int32_t grad_dt, int32_t bits, int32_t block)
{
    if (!dtype_ok(w_dt) || !dtype_ok(grad_dt)) return SLIMFIT_ERR_INVALID_ARG;
    if (bits != 8 && bits != 32) return SLIMFIT_ERR_UNSUPPORTED;
    if (bits == 8 && block != 32 && block != 64 && block != 128 && block != 256) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

int32_t check_workspace(const Layout &lay, const void *ws, size_t bytes)
{
    if (!ws || bytes < lay.bytes) return SLIMFIT_ERR_WORKSPACE;
    if (!aligned_to(ws, 256)) return SLIMFIT_ERR_ALIGNMENT;
    return check_device_range(ws, lay.bytes);
}

int32_t check_step(double lr, double beta1, double beta2, double eps, int64_t step, float floor)
{
    const bool fine = lr >= 0.0 && lr < __builtin_inf() && beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0 && eps > 0.0 && (float)eps > 0.0f &&
                      eps < __builtin_inf() && step >= 1 && step <= 0xFFFFFFFFLL && floor >= 0.0f;
    return fine ? SLIMFIT_OK : SLIMFIT_ERR_INVALID_ARG;
}

Header header_of(int32_t L, const Layout &lay, int32_t w_dt, int32_t grad_dt, int32_t bits, int32_t block)
{
    Header h = {};
    h.magic = kMagic;
    h.n_layers = L;
    h.total_chunks = lay.chunks;
    h.of = lay.of;
    h.w_dt = w_dt;
    h.grad_dt = grad_dt;
    h.bits = bits;
    h.block = bits == 8 ? block : 0;
    return h;
}

template <typename TW, typename TG>
void launch_adamw(int32_t bits, bool score, unsigned grid, hipStream_t st, const char *ws, int32_t L, int64_t chunks, int32_t of, int32_t block, const Step &s,
                  const float *live, const uint8_t *frozen, double *partials)
{
    if (bits == 32 && score) launch(adamw_kernel<TW, TG, 32, true>, grid, kThreads, 0, st, ws, L, chunks, of, block, s, live, frozen, partials);
    else if (bits == 32) launch(adamw_kernel<TW, TG, 32, false>, grid, kThreads, 0, st, ws, L, chunks, of, block, s, live, frozen, partials);
    else if (score) launch(adamw_kernel<TW, TG, 8, true>, grid, kThreads, 0, st, ws, L, chunks, of, block, s, live, frozen, partials);
    else launch(adamw_kernel<TW, TG, 8, false>, grid, kThreads, 0, st, ws, L, chunks, of, block, s, live, frozen, partials);
}

}  // namespace
}  // namespace slimfit

using namespace slimfit;

extern "C" int32_t slimfit_adamw_workspace(int32_t L, const int64_t *numel, size_t *bytes)
{
    if (!bytes) return SLIMFIT_ERR_INVALID_ARG;
    Layout lay;
    const int32_t rc = layout_of(L, numel, &lay);
    if (rc != SLIMFIT_OK) return rc;
    *bytes = lay.bytes;
    return SLIMFIT_OK;
}

extern "C" int32_t slimfit_adamw_plan(void *const *w, int32_t w_dt, const void *const *grad, int32_t grad_dt, void *const *m, void *const *v,
                                      float *const *m_scales, float *const *v_scales, void *const *copies, const float *weight_decay, int32_t bits,
                                      int32_t block, const int64_t *numel, int32_t L, void *workspace, size_t workspace_bytes, void *stream)
{
    StreamScope capture_aware(stream);
    int32_t rc = check_kind(w_dt, grad_dt, bits, block);
    if (rc != SLIMFIT_OK) return rc;
    Layout lay;
    if ((rc = layout_of(L, numel, &lay)) != SLIMFIT_OK) return rc;
    if (L == 0) return SLIMFIT_OK;
    if (!w || !grad || !m || !v || !weight_decay || (bits == 8 && (!m_scales || !v_scales))) return SLIMFIT_ERR_INVALID_ARG;
    if (copies && w_dt != SLIMFIT_F32) return SLIMFIT_ERR_INVALID_ARG;
    // memory of all layers: what is written may be named once only (a tensor of two layers would be stepped by both at once)
    struct Range { uintptr_t at, end; bool written; };
    const std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[(size_t)L * 7 + 1]);
    if (!ranges) return SLIMFIT_ERR_WORKSPACE;
    size_t n_ranges = 0;
    auto apart = [&] {
        std::sort(ranges.get(), ranges.get() + n_ranges, [](const Range &a, const Range &b) { return a.at < b.at; });
        uintptr_t written = 0, any = 0;                     // ends so far
        for (size_t i = 0; i < n_ranges; ++i) {
            const Range &x = ranges[i];
            if (x.at < (x.written ? any : written)) return false;
            any = std::max(any, x.end);
            if (x.written) written = std::max(written, x.end);
        }
        return true;
    };
    for (int pass = 0; pass < 2; ++pass) {                  // what can be told without the runtime comes first
        if (pass == 1 && workspace) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(workspace);
            ranges[n_ranges++] = {at, at + lay.bytes, true};
        }
        if (pass == 1 && !apart()) return SLIMFIT_ERR_INVALID_ARG;
        if (pass == 1 && (rc = check_workspace(lay, workspace, workspace_bytes)) != SLIMFIT_OK) return rc;
        for (int32_t i = 0; i < L; ++i) {
            if (!(weight_decay[i] >= 0.0f) || __builtin_isinf(weight_decay[i])) return SLIMFIT_ERR_INVALID_ARG;
            if (numel[i] == 0) continue;
            const size_t n = (size_t)numel[i], held = bits == 8 ? n : 4 * n, runs = bits == 8 ? 4 * ((n + (size_t)block - 1) / (size_t)block) : 0;
            const struct { const void *p; size_t bytes, align; bool needed; } part[] = {
                {w[i], n * dtype_size(w_dt), 16, true}, {m[i], held, 16, true}, {v[i], held, 16, true},
                {bits == 8 ? m_scales[i] : nullptr, runs, 4, bits == 8}, {bits == 8 ? v_scales[i] : nullptr, runs, 4, bits == 8},
                {copies ? copies[i] : nullptr, 2 * n, 16, false}, {grad[i], n * dtype_size(grad_dt), 16, false}};
            for (const auto &a : part) {
                if (!a.p) {
                    if (a.needed) return SLIMFIT_ERR_INVALID_ARG;
                    continue;
                }
                if (pass == 0 && !aligned_to(a.p, a.align)) return SLIMFIT_ERR_ALIGNMENT;
                if (pass == 0) {
                    const uintptr_t at = reinterpret_cast<uintptr_t>(a.p);
                    ranges[n_ranges++] = {at, at + a.bytes, &a != &part[6]};     // (the gradient is read)
                }
                if (pass == 1 && (rc = check_device_range(a.p, a.bytes)) != SLIMFIT_OK) return rc;
            }
        }
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Header h = header_of(L, lay, w_dt, grad_dt, bits, block);
    int64_t next = 0;
    for (int32_t first = 0; first < L; first += kPlanBatch) {
        PlanBatch batch = {};
        const int count = L - first < kPlanBatch ? L - first : kPlanBatch;
        for (int t = 0; t < count; ++t) {
            const int32_t i = first + t;
            batch.e[t] = Entry{w[i], grad[i], m[i], v[i], bits == 8 ? m_scales[i] : nullptr, bits == 8 ? v_scales[i] : nullptr,
                               copies ? static_cast<uint16_t *>(copies[i]) : nullptr, numel[i], next, weight_decay[i], 0u};
            next += (numel[i] + lay.of - 1) / lay.of;
        }
        launch(plan_kernel, 1, kWave, 0, st, static_cast<char *>(workspace), h, first, count, batch);
    }
    return launch_status();
}

extern "C" int32_t slimfit_adamw_run(const int64_t *numel, int32_t L, int32_t w_dt, int32_t grad_dt, int32_t bits, int32_t block, double lr, double beta1,
                                     double beta2, double eps, int64_t step, float grad_factor, uint32_t seed, const float *live, const uint8_t *frozen,
                                     float floor, float *d_out, void *workspace, size_t workspace_bytes, void *stream)
{
    StreamScope capture_aware(stream);
    int32_t rc = check_kind(w_dt, grad_dt, bits, block);
    if (rc != SLIMFIT_OK) return rc;
    if ((rc = check_step(lr, beta1, beta2, eps, step, floor)) != SLIMFIT_OK) return rc;
    Layout lay;
    if ((rc = layout_of(L, numel, &lay)) != SLIMFIT_OK) return rc;
    if (L == 0) return SLIMFIT_OK;
    if (!aligned_to(d_out, 4) || !aligned_to(live, 4)) return SLIMFIT_ERR_ALIGNMENT;
    if (workspace) {
        const size_t d_bytes = d_out ? sizeof(float) * (size_t)L : 0, live_bytes = live ? 3 * sizeof(float) : 0, frozen_bytes = frozen ? (size_t)L : 0;
        auto shares = [](const void *a, size_t a_bytes, const void *b, size_t b_bytes) { return a_bytes > 0 && b_bytes > 0 && meet(a, a_bytes, b, b_bytes); };
        if (shares(workspace, lay.bytes, d_out, d_bytes) || shares(workspace, lay.bytes, live, live_bytes) || shares(workspace, lay.bytes, frozen, frozen_bytes) ||
            shares(d_out, d_bytes, live, live_bytes) || shares(d_out, d_bytes, frozen, frozen_bytes))
            return SLIMFIT_ERR_INVALID_ARG;
    }
    if ((rc = check_workspace(lay, workspace, workspace_bytes)) != SLIMFIT_OK) return rc;
    if (d_out && (rc = check_device_range(d_out, sizeof(float) * (size_t)L)) != SLIMFIT_OK) return rc;
    if (live && (rc = check_device_range(live, 3 * sizeof(float))) != SLIMFIT_OK) return rc;
    if (frozen && (rc = check_device_range(frozen, (size_t)L)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const char *ws = static_cast<const char *>(workspace);
    double *partials = reinterpret_cast<double *>(static_cast<char *>(workspace) + table_bytes(L));
    const uint32_t t = (uint32_t)step;
    const Step s = {beta1, beta2, (float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, (float)lr,
                    (float)(lr / (1.0 - power(beta1, t))), (float)(1.0 / __builtin_sqrt(1.0 - power(beta2, t))), grad_factor, floor, seed, t};
    const Header want = header_of(L, lay, w_dt, grad_dt, bits, block);
    if (lay.chunks > 0) {
        const unsigned grid = (unsigned)lay.chunks;
        if (w_dt == SLIMFIT_F32 && grad_dt == SLIMFIT_F32)
            launch_adamw<float, float>(bits, d_out != nullptr, grid, st, ws, L, lay.chunks, lay.of, want.block, s, live, frozen, partials);
        else if (w_dt == SLIMFIT_F32)
            launch_adamw<float, uint16_t>(bits, d_out != nullptr, grid, st, ws, L, lay.chunks, lay.of, want.block, s, live, frozen, partials);
        else if (grad_dt == SLIMFIT_F32)
            launch_adamw<uint16_t, float>(bits, d_out != nullptr, grid, st, ws, L, lay.chunks, lay.of, want.block, s, live, frozen, partials);
        else
            launch_adamw<uint16_t, uint16_t>(bits, d_out != nullptr, grid, st, ws, L, lay.chunks, lay.of, want.block, s, live, frozen, partials);
    }
    if (d_out) launch(finish_kernel, (unsigned)L, kThreads, 0, st, ws, L, lay.chunks, want, partials, d_out);
    return launch_status();
}

extern "C" int32_t slimfit_adamw_states(const uint8_t *m, const float *m_scales, const uint8_t *v, const float *v_scales, int64_t n, int32_t block,
                                        float *m_out, float *v_out, void *stream)
{
    StreamScope capture_aware(stream);
    if (n < 0) return SLIMFIT_ERR_INVALID_ARG;
    if (block != 32 && block != 64 && block != 128 && block != 256) return SLIMFIT_ERR_UNSUPPORTED;
    if (n > ((int64_t)1 << 40)) return SLIMFIT_ERR_UNSUPPORTED;
    if (n == 0) return SLIMFIT_OK;
    if (!m || !m_scales || !v || !v_scales || !m_out || !v_out) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(m, 16) || !aligned_to(v, 16) || !aligned_to(m_out, 16) || !aligned_to(v_out, 16) || !aligned_to(m_scales, 4) || !aligned_to(v_scales, 4))
        return SLIMFIT_ERR_ALIGNMENT;
    const size_t codes = (size_t)n, scales = 4 * (((size_t)n + (size_t)block - 1) / (size_t)block), out = 4 * (size_t)n;
    if (meet(m_out, out, v_out, out)) return SLIMFIT_ERR_INVALID_ARG;
    for (float *o : {m_out, v_out})
        if (meet(o, out, m, codes) || meet(o, out, v, codes) || meet(o, out, m_scales, scales) || meet(o, out, v_scales, scales)) return SLIMFIT_ERR_INVALID_ARG;
    int32_t rc;
    if ((rc = check_device_range(m, codes)) != SLIMFIT_OK || (rc = check_device_range(v, codes)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(m_scales, scales)) != SLIMFIT_OK || (rc = check_device_range(v_scales, scales)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(m_out, out)) != SLIMFIT_OK || (rc = check_device_range(v_out, out)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    constexpr int64_t kMost = kMaxGridThreads * kStates, kPass = kThreads * kStates;
    for (int64_t first = 0; first < n; first += kMost) {
        const int64_t left = n - first < kMost ? n - first : kMost;
        launch(states_kernel, (unsigned)((left + kPass - 1) / kPass), kThreads, 0, st, m, m_scales, v, v_scales, n, __builtin_ctz((unsigned)block), m_out, v_out,
               first);
    }
    return launch_status();
}
