// Gated activations around the low-bit cache of their input (not in the paper, whose feed-forward layers have a plain
// GELU; its placement, 4 or 8 bits for the activation's input, carried over to the layers of decoder models): rows x =
// [g | u] of 2 F elements,
//     y = act(g) * u,      dx = [dy * u^ * act'(g^) | dy * act(g^)],
// act the logistic one (g / (1 + e^-g)) or GELU, and g^, u^ what the cache of x gives back.
//
// Layout: vector i of the rows of y (16 bytes) is a lane's; it holds the two vectors of x that belong to it, F elements
// apart, so that x is read once for the product and for both of its quantisation blocks.  F is a multiple of the block:
// blocks lie in one half of one row, and block / V consecutive lanes hold one, as in the quantiser, whose codes and scales
// these are bit for bit.
//
// Bound by HBM: 16384 x 2 x 4096 bf16 with 8 bits 88 us forward (545 MB, 6.2 TB/s, the card's 1 : 1 stream) and 82 backward (545 MB);
// 7289 x 2 x 2048 fp32 with 4 bits and GELU 32 and 31 (196 MB each); a single row of 4096 2.0 us, the launch.
#include "elements.hpp"

namespace slimfit {
namespace {

constexpr int kThreads = 128;
constexpr int kThreadsB = 256;
constexpr int kUnroll = 2;                 // vectors of y a lane: four blocks, whose divisions a quad of lanes shares
constexpr int kUnrollB = 1;

// 1 / (1 + e^-x): e^-x overflows to infinity below -88, where the quotient is 0 (its value there is below 2^-126)
__device__ __forceinline__ float logistic(float x)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504088896340736f));
}
// erfc's argument is held at 6, the polynomial's least value (8e-15): held at 4.2 it would leave GELU 1.5e-9 of the gate, however far
// below zero that is (setting it to 0 there instead: 7289 x 2 x 2048 fp32 forward and backward 65.6 -> 67.3 us).
constexpr float kFar = 6.0f;
template <bool GELU>
__device__ __forceinline__ float act_value(float x) { return GELU ? (0.5f * x) * twice_normal_cdf(x, kFar) : x * logistic(x); }
// act(x) and act'(x)
template <bool GELU>
__device__ __forceinline__ void act_both(float x, float &value, float &slope)
{
    if (GELU) {
        const float cdf = 0.5f * twice_normal_cdf(x, kFar);
        value = x * cdf;
        slope = cdf + x * (__builtin_amdgcn_exp2f(((-0.5f * x) * x) * 1.44269504088896340736f) * 0.39894228040143267794f);
    } else {
        const float p = logistic(x);
        value = x * p;
        slope = p * fmaf(x, 1.0f - p, 1.0f);
    }
}

// BITS 0: nothing is kept.  G: lanes a block (0: one factor for all).
template <typename T, int BITS, int G, bool GELU>
__global__ __launch_bounds__(kThreads) void gated_kernel(const T *__restrict__ x, uint32_t vectors, uint32_t across, Divide row_of, float fixed_mult,
                                                         T *__restrict__ y, uint8_t *__restrict__ codes, float *__restrict__ scales)
{
    using raw = typename Vec<T>::raw;
    constexpr int V = Vec<T>::V;
    const uint32_t first = blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
    float f[2 * kUnroll][V];                               // gate and up of each of the lane's vectors
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const uint32_t i = first + u * kThreads;
        raw g{}, w{};
        if (i < vectors) {
            const int64_t at = (int64_t)i + (int64_t)row_of(i) * across;
            g = load_global<true>(reinterpret_cast<const raw *>(x) + at);
            w = load_global<true>(reinterpret_cast<const raw *>(x) + at + across);
        }
        Vec<T>::unpack(g, f[2 * u]);
        Vec<T>::unpack(w, f[2 * u + 1]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const uint32_t i = first + u * kThreads;
        float out[V];
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = act_value<GELU>(f[2 * u][e]) * f[2 * u + 1][e];
        if (i < vectors) store_global<true>(reinterpret_cast<raw *>(y) + i, Vec<T>::pack(out));
    }
    if constexpr (BITS != 0) {
        float mult[2 * kUnroll];
#pragma unroll
        for (int b = 0; b < 2 * kUnroll; ++b) mult[b] = fixed_mult;
        if constexpr (G != 0) {
            uint32_t a[2 * kUnroll];
#pragma unroll
            for (int b = 0; b < 2 * kUnroll; ++b) {
                float m = 0.0f;
#pragma unroll
                for (int e = 0; e < V; ++e) m = fmaxf(m, fabsf(f[b][e]));
                a[b] = group_max_u32(__builtin_bit_cast(uint32_t, m), G);
            }
            float scale;
            quad_scales<BITS, 2 * kUnroll>(a, (int)threadIdx.x, mult, scale);
            const int own = threadIdx.x & (G - 1);         // lanes 0 .. 3 of a group store a block's scale each
            const uint32_t i = first + (own >> 1) * kThreads;
            if (own < 2 * kUnroll && i < vectors)
                scales[((int64_t)i + (int64_t)row_of(i) * across + (own & 1) * across) / G] = scale;
        }
#pragma unroll
        for (int b = 0; b < 2 * kUnroll; ++b) {
            const uint32_t i = first + (b >> 1) * kThreads;
            uint32_t w[2];
            pack_codes<BITS, V>(f[b], mult[b], w);
            if (i < vectors) {
                constexpr int BYTES = V * BITS / 8;
                uint8_t *dst = codes + ((int64_t)i + (int64_t)row_of(i) * across + (b & 1) * across) * BYTES;
                if (BYTES == 2) store_global<true>(reinterpret_cast<uint16_t *>(dst), (uint16_t)w[0]);
                else if (BYTES == 4) store_global<true>(reinterpret_cast<uint32_t *>(dst), w[0]);
                else store_global<true>(reinterpret_cast<u32x2 *>(dst), u32x2{w[0], w[1]});
            }
        }
    }
}

template <typename T, int BITS, bool BLOCKED, bool GELU>
__global__ __launch_bounds__(kThreadsB) void gated_backward_kernel(const uint8_t *__restrict__ codes, const float *__restrict__ scales, uint32_t vectors,
                                                                   uint32_t across, Divide row_of, int block_shift, float fixed_step,
                                                                   const T *__restrict__ dy, T *__restrict__ dx)
{
    using raw = typename Vec<T>::raw;
    constexpr int V = Vec<T>::V, BYTES = V * BITS / 8;
    const uint32_t first = blockIdx.x * (kThreadsB * kUnrollB) + threadIdx.x;
    uint32_t w[2 * kUnrollB][2];
    float step[2 * kUnrollB];
    raw grad[kUnrollB];
#pragma unroll
    for (int u = 0; u < kUnrollB; ++u) {
        const uint32_t i = first + u * kThreadsB;
        if (i >= vectors) continue;
        grad[u] = load_global<true>(reinterpret_cast<const raw *>(dy) + i);
        const int64_t at = (int64_t)i + (int64_t)row_of(i) * across;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t(&to)[2] = w[2 * u + h];
            const uint8_t *src = codes + (at + h * across) * BYTES;
            to[1] = 0u;
            if (BYTES == 2) to[0] = load_global<true>(reinterpret_cast<const uint16_t *>(src));
            else if (BYTES == 4) to[0] = load_global<true>(reinterpret_cast<const uint32_t *>(src));
            else { const u32x2 t = load_global<true>(reinterpret_cast<const u32x2 *>(src)); to[0] = t.x; to[1] = t.y; }
            step[2 * u + h] = BLOCKED ? scales[(at + h * across) >> block_shift] : fixed_step;
        }
    }
#pragma unroll
    for (int u = 0; u < kUnrollB; ++u) {
        const uint32_t i = first + u * kThreadsB;
        if (i >= vectors) continue;
        float d[V], dg[V], du[V];
        Vec<T>::unpack(grad[u], d);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float g = (float)code_field<BITS>(w[2 * u][e * BITS / 32], e % (32 / BITS)) * step[2 * u];
            const float up = (float)code_field<BITS>(w[2 * u + 1][e * BITS / 32], e % (32 / BITS)) * step[2 * u + 1];
            float value, slope;
            act_both<GELU>(g, value, slope);
            dg[e] = d[e] * up * slope;
            du[e] = d[e] * value;
        }
        raw *to = reinterpret_cast<raw *>(dx) + ((int64_t)i + (int64_t)row_of(i) * across);
        store_global<true>(to, Vec<T>::pack(dg));
        store_global<true>(to + across, Vec<T>::pack(du));
    }
}

// Rows of one launch: vectors are counted in 31 bits
inline int64_t rows_of_launch(int64_t across) { return ((int64_t)1 << 30) / across; }

template <typename T, int BITS, bool GELU>
void launch_gated(const void *x, int64_t rows, int64_t F, int mode, int block, int frac_bits, void *y, uint8_t *codes, float *scales, hipStream_t st)
{
    constexpr int V = Vec<T>::V;
    const int64_t across = F / V, most = rows_of_launch(across);
    const Divide row_of((uint32_t)across);
    for (int64_t r = 0; r < rows; r += most) {
        const uint32_t vectors = (uint32_t)((rows - r < most ? rows - r : most) * across);
        const dim3 grid((vectors + kThreads * kUnroll - 1) / (kThreads * kUnroll)), tb(kThreads);
        const T *xp = static_cast<const T *>(x) + r * 2 * F;
        T *yp = static_cast<T *>(y) + r * F;
        uint8_t *cp = BITS ? codes + r * 2 * F * BITS / 8 : nullptr;
        float *sp = BITS && mode == SLIMFIT_Q_BLOCK ? scales + r * 2 * F / block : nullptr;
        const int G = BITS && mode == SLIMFIT_Q_BLOCK ? block / V : 0;
        const float mult = BITS && mode == SLIMFIT_Q_FIXED ? __builtin_ldexpf(1.0f, frac_bits) : 0.0f;
        if constexpr (BITS != 0) {
            switch (G) {
            case 4: launch(gated_kernel<T, BITS, 4, GELU>, grid, tb, 0, st, xp, vectors, (uint32_t)across, row_of, mult, yp, cp, sp); continue;
            case 8: launch(gated_kernel<T, BITS, 8, GELU>, grid, tb, 0, st, xp, vectors, (uint32_t)across, row_of, mult, yp, cp, sp); continue;
            case 16: launch(gated_kernel<T, BITS, 16, GELU>, grid, tb, 0, st, xp, vectors, (uint32_t)across, row_of, mult, yp, cp, sp); continue;
            case 32: launch(gated_kernel<T, BITS, 32, GELU>, grid, tb, 0, st, xp, vectors, (uint32_t)across, row_of, mult, yp, cp, sp); continue;
            case 64: launch(gated_kernel<T, BITS, 64, GELU>, grid, tb, 0, st, xp, vectors, (uint32_t)across, row_of, mult, yp, cp, sp); continue;
            default: break;
            }
        }
        launch(gated_kernel<T, BITS, 0, GELU>, grid, tb, 0, st, xp, vectors, (uint32_t)across, row_of, mult, yp, cp, sp);
    }
}

template <typename T, int BITS, bool GELU>
void launch_gated_backward(const uint8_t *codes, const float *scales, int64_t rows, int64_t F, int mode, int block, int frac_bits, const void *dy,
                           void *dx, hipStream_t st)
{
    constexpr int V = Vec<T>::V;
    const int64_t across = F / V, most = rows_of_launch(across);
    const Divide row_of((uint32_t)across);
    for (int64_t r = 0; r < rows; r += most) {
        const uint32_t vectors = (uint32_t)((rows - r < most ? rows - r : most) * across);
        const dim3 grid((vectors + kThreadsB * kUnrollB - 1) / (kThreadsB * kUnrollB)), tb(kThreadsB);
        const T *gp = static_cast<const T *>(dy) + r * F;
        T *dp = static_cast<T *>(dx) + r * 2 * F;
        const uint8_t *cp = codes + r * 2 * F * BITS / 8;
        if (mode == SLIMFIT_Q_FIXED)
            launch(gated_backward_kernel<T, BITS, false, GELU>, grid, tb, 0, st, cp, nullptr, vectors, (uint32_t)across, row_of, 0,
                   __builtin_ldexpf(1.0f, -frac_bits), gp, dp);
        else
            launch(gated_backward_kernel<T, BITS, true, GELU>, grid, tb, 0, st, cp, scales + r * 2 * F / block, vectors, (uint32_t)across, row_of,
                   __builtin_ctz((unsigned)(block / V)), 0.0f, gp, dp);
    }
}

int32_t validate(int32_t dt, int64_t rows, int64_t F, int32_t act, int32_t mode, int32_t bits, int32_t block, int32_t frac_bits)
{
    if (!dtype_ok(dt) || rows < 0 || F < 0) return SLIMFIT_ERR_INVALID_ARG;
    if (act != SLIMFIT_ACT_SILU && act != SLIMFIT_ACT_GELU) return SLIMFIT_ERR_INVALID_ARG;
    if (bits != 0) {
        if (mode != SLIMFIT_Q_FIXED && mode != SLIMFIT_Q_BLOCK) return SLIMFIT_ERR_INVALID_ARG;
        if (bits != 4 && bits != 8) return SLIMFIT_ERR_UNSUPPORTED;
        if (mode == SLIMFIT_Q_FIXED && (frac_bits < -32 || frac_bits > 32)) return SLIMFIT_ERR_UNSUPPORTED;
        if (mode == SLIMFIT_Q_BLOCK && block != 32 && block != 64 && block != 128 && block != 256) return SLIMFIT_ERR_UNSUPPORTED;
        if (mode == SLIMFIT_Q_BLOCK && F % block != 0) return SLIMFIT_ERR_UNSUPPORTED;
    }
    if (F % (dt == SLIMFIT_F32 ? 4 : 8) != 0) return SLIMFIT_ERR_UNSUPPORTED;
    if (F > ((int64_t)1 << 24) || (F > 0 && rows > ((int64_t)1 << 40) / F)) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

}  // namespace
}  // namespace slimfit

using namespace slimfit;

extern "C" int32_t slimfit_gated_quant_pack(const void *x, int32_t dt, int64_t rows, int64_t F, int32_t act, int32_t mode, int32_t bits,
                                            int32_t block, int32_t frac_bits, void *y, uint8_t *codes, float *scales, void *stream)
{
    StreamScope capture_aware(stream);
    int32_t rc = validate(dt, rows, F, act, mode, bits, block, frac_bits);
    if (rc != SLIMFIT_OK) return rc;
    if (rows == 0 || F == 0) return SLIMFIT_OK;
    const bool blocked = bits != 0 && mode == SLIMFIT_Q_BLOCK;
    if (!x || !y || (bits != 0 && !codes) || (blocked && !scales)) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(x, 16) || !aligned_to(y, 16) || (bits != 0 && !aligned_to(codes, 16)) || (blocked && !aligned_to(scales, 16)))
        return SLIMFIT_ERR_ALIGNMENT;
    const size_t n = (size_t)rows * (size_t)F, e = dtype_size(dt);
    if (meet(x, 2 * n * e, y, n * e)) return SLIMFIT_ERR_INVALID_ARG;
    if ((rc = check_device_range(x, 2 * n * e)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(y, n * e)) != SLIMFIT_OK) return rc;
    if (bits != 0 && (rc = check_device_range(codes, 2 * n * (size_t)bits / 8)) != SLIMFIT_OK) return rc;
    if (blocked && (rc = check_device_range(scales, 2 * n / (size_t)block * 4)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool gelu = act == SLIMFIT_ACT_GELU;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (bits == 0) gelu ? launch_gated<T, 0, true>(x, rows, F, mode, block, frac_bits, y, codes, scales, st)
                            : launch_gated<T, 0, false>(x, rows, F, mode, block, frac_bits, y, codes, scales, st);
        else if (bits == 4) gelu ? launch_gated<T, 4, true>(x, rows, F, mode, block, frac_bits, y, codes, scales, st)
                                 : launch_gated<T, 4, false>(x, rows, F, mode, block, frac_bits, y, codes, scales, st);
        else gelu ? launch_gated<T, 8, true>(x, rows, F, mode, block, frac_bits, y, codes, scales, st)
                  : launch_gated<T, 8, false>(x, rows, F, mode, block, frac_bits, y, codes, scales, st);
    };
    if (dt == SLIMFIT_F32) go(float{});
    else go(uint16_t{});
    return launch_status();
}

extern "C" int32_t slimfit_gated_backward_dequant(const uint8_t *codes, const float *scales, int64_t rows, int64_t F, int32_t act, int32_t mode,
                                                  int32_t bits, int32_t block, int32_t frac_bits, const void *dy, void *dx, int32_t dt,
                                                  void *stream)
{
    StreamScope capture_aware(stream);
    if (bits == 0) return SLIMFIT_ERR_UNSUPPORTED;
    int32_t rc = validate(dt, rows, F, act, mode, bits, block, frac_bits);
    if (rc != SLIMFIT_OK) return rc;
    if (rows == 0 || F == 0) return SLIMFIT_OK;
    const bool blocked = mode == SLIMFIT_Q_BLOCK;
    if (!dy || !dx || !codes || (blocked && !scales)) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(dy, 16) || !aligned_to(dx, 16) || !aligned_to(codes, 16) || (blocked && !aligned_to(scales, 16))) return SLIMFIT_ERR_ALIGNMENT;
    const size_t n = (size_t)rows * (size_t)F, e = dtype_size(dt);
    if (meet(dx, 2 * n * e, dy, n * e)) return SLIMFIT_ERR_INVALID_ARG;
    if ((rc = check_device_range(dx, 2 * n * e)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(dy, n * e)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(codes, 2 * n * (size_t)bits / 8)) != SLIMFIT_OK) return rc;
    if (blocked && (rc = check_device_range(scales, 2 * n / (size_t)block * 4)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const bool gelu = act == SLIMFIT_ACT_GELU;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (bits == 4) gelu ? launch_gated_backward<T, 4, true>(codes, scales, rows, F, mode, block, frac_bits, dy, dx, st)
                            : launch_gated_backward<T, 4, false>(codes, scales, rows, F, mode, block, frac_bits, dy, dx, st);
        else gelu ? launch_gated_backward<T, 8, true>(codes, scales, rows, F, mode, block, frac_bits, dy, dx, st)
                  : launch_gated_backward<T, 8, false>(codes, scales, rows, F, mode, block, frac_bits, dy, dx, st);
    };
    if (dt == SLIMFIT_F32) go(float{});
    else go(uint16_t{});
    return launch_status();
}
