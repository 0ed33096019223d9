// Weight gradient of an active linear layer straight from the low-bit cache of its input (Alg. 4's dW = dY^T X with X as the
// cache gives it back): dw[n][k] = sum over m of dy[m][n] code[m][k] scale[m][k / block].
//
// Both operands lie across the sum.  Their rows go to LDS as they lie, 32 rows of the sum a step, the codes as bf16, and the reads turn
// them (ds_read_b64_tr_b16): a lane gets eight rows of one column, which is what it hands to v_mfma_f32_16x16x32_bf16.
//   bf16  x^ = code * scale rounded to bf16, as the cache gives it to a bf16 tensor: one product, where x^ in fp32 would take two.  The
//         result is off by 0.0021 of its norm, by 0.0017 if x^ were not rounded (its own rounding to bf16).
//   fp32  the scale goes onto dy (a tile lies in one block), whose product is rounded to fp32 once and taken apart exactly
//         into three bf16 numbers; the codes are whole numbers that bf16 holds.  Three products in place of the six that two
//         fp32 operands take.
// Rows past M are read as zeros by the bounds of the buffer descriptors, which move along with the steps.  Where there are
// fewer tiles than the compute units can hold, the rows are shared out and the parts added up in order by a second kernel.
//
// 4096 x 1024 over 16384 bf16 rows 160 to 190 us with the parts' sum (the card's clock follows its load: short bursts are the faster
// ones), 720 to 860 TFLOP/s; torch's product of the same sizes, x^ in memory as bf16, takes 200, and a product of 8192^3 runs at 1240.
// 1024 x 4096 over 12608 fp32 rows 394 to 447 us, 240 to 270 TFLOP/s; torch's fp32 product 750.  What bounds it is how far loading,
// forming operands and multiplying overlap: without the loads 149 of 194 us, without forming operands 134, with operands of
// zeros 158 (fp32 342, 255 and 421 of 470).  Tried and no faster at that size: two LDS stages with loads one and two steps ahead
// (184 and 187), two groups of four waves that form and multiply in turn (190 to 197), operands turned in registers on the
// way in (247); fp32 alike (465 to 490), its single stage with four workgroups a compute unit 431.
#include "common.hpp"
#include "weight_plan.hpp"

#include <type_traits>

namespace slimfit {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void *at, int64_t bytes)      // bytes from `at` to the matrix's end; reads past it give 0
{
    const int64_t most = 0xFFFFFFF0LL, n = bytes < 0 ? 0 : bytes < most ? bytes : most;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, (int)(uint32_t)n, 0x00020000);
}

// A tile of dw is TN x TK, a step 32 rows of the sum.  WAVES_N x WAVES_K waves.
template <typename T, int TN, int TK> struct Config;
template <> struct Config<uint16_t, 256, 128> { static constexpr int PARTS = 1, WAVES_N = 2; };
template <> struct Config<uint16_t, 128, 128> { static constexpr int PARTS = 1, WAVES_N = 2; };
template <> struct Config<float, 128, 64> { static constexpr int PARTS = 3, WAVES_N = 4; };
template <> struct Config<float, 128, 32> { static constexpr int PARTS = 3, WAVES_N = 4; };

// a row of a tile in LDS: 32 bytes more than it holds, so that sixteen rows' 32 bytes, which a transposing read takes, are in
// different banks two by two
constexpr int pitch_of(int columns) { return columns * 2 + 32; }

struct Sizes {
    int64_t M, N, K, split_rows;           // split_rows: rows of a part, a multiple of the step
    int tiles_n, tiles_k, splits, block_shift;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 *LdsVector;
// eight rows of one column, from a tile whose rows lie along the columns: rows 4 g .. 4 g + 3 and 16 + 4 g .. of the step for the lanes
// of group g = lane / 16 (the order of the sum is the same for both operands, so any is), column lane % 16 of sixteen
template <int PITCH>
__device__ __forceinline__ bf16x8 fragment(const char *at)
{
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVector)(at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVector)(at + 16 * PITCH));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// How dy is read, 16 bytes a thread: its rows begin on 16 bytes; they begin anywhere, and the last vector of a row is the one that ends
// with it; or (rows shorter than a vector) element by element.
enum Rows { kAligned, kAnywhere, kShort };

template <typename T, int BITS, int TN, int TK, Rows ROWS>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 5 : 2)
weight_kernel(const T *__restrict__ dy, const uint8_t *__restrict__ codes, const float *__restrict__ scales, T *__restrict__ dw,
              float *__restrict__ parts, Sizes z)
{
    using C = Config<T, TN, TK>;
    constexpr int PARTS = C::PARTS, WAVES_N = C::WAVES_N, WAVES_K = 4 / WAVES_N, FN = TN / WAVES_N / 16, FK = TK / WAVES_K / 16;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int E = 16 / sizeof(T);                      // elements of dy a thread takes at a time
    constexpr int LINE = TN / E, LINES = kThreads / LINE, PASSES = kStep / LINES;
    constexpr int CODES = kStep * TK / kThreads;           // codes a thread takes, of one row
    constexpr int PY = pitch_of(TN), PX = pitch_of(TK), PART = kStep * PY, STAGE = PARTS * PART + kStep * PX;
    __shared__ __align__(16) char stage[STAGE];
    const int t = threadIdx.x, lane = t & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(t >> 6);
    // Workgroups go to the eight XCDs in turn; an XCD's take bands of four tile rows, column by column, of one part of the sum
    const int tiles = z.tiles_n * z.tiles_k, all = tiles * z.splits;
    const int each = all / 8, b0 = (int)blockIdx.x, turn = b0 < each * 8 ? (b0 % 8) * each + b0 / 8 : b0;
    const int split = turn / tiles, id = turn % tiles;
    const int band = id / (4 * z.tiles_k), in_band = id % (4 * z.tiles_k), height = min(4, z.tiles_n - 4 * band);
    const int64_t n0 = (int64_t)(band * 4 + in_band % height) * TN, k0 = (int64_t)(in_band / height) * TK;
    const int64_t m0 = (int64_t)split * z.split_rows, m1 = min(m0 + z.split_rows, z.M);
    const int steps = m1 > m0 ? (int)((m1 - m0 + kStep - 1) / kStep) : 0;

    const int64_t dy_row = z.N * (int64_t)sizeof(T), code_row = z.K * BITS / 8, scale_row = (z.K >> z.block_shift) * 4;
    const int ny = t % LINE * E, my = t / LINE, kx = t % (TK / CODES) * CODES, mx = t / (TK / CODES);
    int at_dy[PASSES], at_scale[F32 ? PASSES : 1];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) at_dy[p] = (int)((p * LINES + my) * dy_row + (ROWS == kAnywhere ? min(n0 + ny, z.N - E) : n0 + ny) * (int64_t)sizeof(T));
    // columns by which the thread's vector begins before its place (past the row's end it does not matter where)
    const int before = ROWS == kAnywhere && n0 + ny < z.N ? (int)(n0 + ny - min(n0 + ny, z.N - E)) : 0;
    const int at_code = (int)(mx * code_row + (k0 + kx) * BITS / 8);
    if constexpr (F32) {                                   // (the tile lies in one block)
#pragma unroll
        for (int p = 0; p < PASSES; ++p) at_scale[p] = (int)((p * LINES + my) * scale_row + (k0 >> z.block_shift) * 4);
    } else {
        at_scale[0] = (int)(mx * scale_row + ((k0 + kx) >> z.block_shift) * 4);
    }

    struct Held {
        u32x4 y[PASSES];
        uint32_t c[CODES * BITS >= 32 ? CODES * BITS / 32 : 1];
        float s[F32 ? PASSES : 1];
    } held;
    auto load = [&](int64_t m) {
        const Buffer by = buffer_of(reinterpret_cast<const char *>(dy) + m * dy_row, (z.M - m) * dy_row);
        const Buffer bc = buffer_of(codes + m * code_row, (z.M - m) * code_row);
        const Buffer bs = buffer_of(reinterpret_cast<const char *>(scales) + m * scale_row, (z.M - m) * scale_row);
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            if constexpr (ROWS != kShort) {
                const auto v = __builtin_amdgcn_raw_buffer_load_b128(by, at_dy[p], 0, 0);
                held.y[p] = u32x4{v[0], v[1], v[2], v[3]};
            } else if constexpr (F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i) held.y[p][i] = __builtin_amdgcn_raw_buffer_load_b32(by, at_dy[p] + 4 * i, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    held.y[p][i] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(by, at_dy[p] + 4 * i, 0, 0) |
                                   (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(by, at_dy[p] + 4 * i + 2, 0, 0) << 16;
            }
        }
        constexpr int BYTES = CODES * BITS / 8;
        if constexpr (BYTES == 16) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b128(bc, at_code, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) held.c[i] = v[i];
        } else if constexpr (BYTES == 8) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(bc, at_code, 0, 0);
            held.c[0] = v[0];
            held.c[1] = v[1];
        } else if constexpr (BYTES == 4) {
            held.c[0] = __builtin_amdgcn_raw_buffer_load_b32(bc, at_code, 0, 0);
        } else {
            held.c[0] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(bc, at_code, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < (F32 ? PASSES : 1); ++i) {
            const uint32_t v = __builtin_amdgcn_raw_buffer_load_b32(bs, at_scale[i], 0, 0);
            held.s[i] = __builtin_bit_cast(float, v);
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            char *to = stage + (p * LINES + my) * PY + ny * 2;
            auto put = [&](char *at, const auto &words, auto n) {          // n words of two columns each
                constexpr int W = decltype(n)::value;
                if (ROWS == kAnywhere && before != 0) {    // those of its columns that are in its place; the thread before it has the others
#pragma unroll
                    for (int i = 0; i < 2 * W; ++i)
                        if (i >= before) reinterpret_cast<uint16_t *>(at)[i - before] = (uint16_t)(words[i / 2] >> (i % 2 * 16));
                } else if constexpr (W == 4) {
                    *reinterpret_cast<u32x4 *>(at) = u32x4{words[0], words[1], words[2], words[3]};
                } else {
                    *reinterpret_cast<u32x2 *>(at) = u32x2{words[0], words[1]};
                }
            };
            if constexpr (!F32) {
                put(to, held.y[p], std::integral_constant<int, 4>{});
            } else {
                uint32_t h[2], m[2], l[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t u = held.y[p][2 * i], v = held.y[p][2 * i + 1];
                    float a = __builtin_bit_cast(float, u) * held.s[p], b = __builtin_bit_cast(float, v) * held.s[p];
                    h[i] = bf16_narrow2(a, b);
                    a -= __builtin_bit_cast(float, h[i] << 16);
                    b -= __builtin_bit_cast(float, h[i] & 0xFFFF0000u);
                    m[i] = bf16_narrow2(a, b);
                    a -= __builtin_bit_cast(float, m[i] << 16);
                    b -= __builtin_bit_cast(float, m[i] & 0xFFFF0000u);
                    l[i] = bf16_narrow2(a, b);
                }
                put(to, h, std::integral_constant<int, 2>{});
                put(to + PART, m, std::integral_constant<int, 2>{});
                put(to + 2 * PART, l, std::integral_constant<int, 2>{});
            }
        }
        uint32_t x[CODES / 2];
#pragma unroll
        for (int i = 0; i < CODES; i += 2) {
            float a = (float)code_field<BITS>(held.c[i * BITS / 32], i % (32 / BITS)), b = (float)code_field<BITS>(held.c[i * BITS / 32], i % (32 / BITS) + 1);
            if constexpr (!F32) {
                a *= held.s[0];
                b *= held.s[0];
            }
            x[i / 2] = bf16_narrow2(a, b);
        }
        char *to = stage + PARTS * PART + mx * PX + kx * 2;
        if constexpr (CODES >= 8) {
#pragma unroll
            for (int i = 0; i < CODES / 8; ++i) reinterpret_cast<u32x4 *>(to)[i] = u32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
        } else {
            *reinterpret_cast<u32x2 *>(to) = u32x2{x[0], x[1]};
        }
    };

    f32x4 acc[FK][FN];
#pragma unroll
    for (int i = 0; i < FK; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int wn = wave / WAVES_K * (TN / WAVES_N), wk = wave % WAVES_K * (TK / WAVES_K);
    const int place = 4 * (lane >> 4) + (lane & 15) / 4, column = (lane & 3) * 4;      // of the lane's first four elements
    const int read_y = place * PY + (wn + column) * 2, read_x = PARTS * PART + place * PX + (wk + column) * 2;
    load(m0);
    for (int s = 0; s < steps; ++s) {
        store();
        load(m0 + (int64_t)(s + 1) * kStep);           // past the last step: the next part's rows, or zeros
        __syncthreads();
        __builtin_amdgcn_s_setprio(1);                      // 1 to 2 % of the time
        bf16x8 fx[FK];
#pragma unroll
        for (int i = 0; i < FK; ++i) fx[i] = fragment<PX>(stage + read_x + i * 32);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) {         // small parts first
                const bf16x8 fy = fragment<PY>(stage + read_y + p * PART + j * 32);
#pragma unroll
                for (int i = 0; i < FK; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[i], fy, acc[i][j], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        __syncthreads();
    }
    float *const sums = parts ? parts + (int64_t)split * z.N * z.K : F32 ? reinterpret_cast<float *>(dw) : nullptr;
    bool odd = false;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t n = n0 + wn + j * 16 + (lane & 15);
        if (n >= z.N) continue;
#pragma unroll
        for (int i = 0; i < FK; ++i) {
            const int64_t k = k0 + wk + i * 16 + (lane >> 4) * 4;
            if (k >= z.K) continue;
            const f32x4 v = acc[i][j];
            if (F32 || parts) *reinterpret_cast<f32x4 *>(sums + n * z.K + k) = v;
            else *reinterpret_cast<u32x2 *>(dw + n * z.K + k) = u32x2{bf16_narrow2(v[0], v[1]), bf16_narrow2(v[2], v[3])};
            if constexpr (F32) {
#pragma unroll
                for (int q = 0; q < 4; ++q) odd |= !(__builtin_fabsf(v[q]) < __builtin_inff());
            }
        }
    }
    if constexpr (F32) {
        // dy * scale that is infinite, NaN or rounds to bf16's infinity, or a sum that overflows: what comes out there is what the fp32
        // matrix instructions make of dy and x^, for which the wave goes over its share of the tile again (12608 x 1024 x 4096 with all
        // entries of dy NaN 3.0 ms in all).  Five waves a SIMD are asked for, or the compiler spends the registers that this leaves unused.
        if (__builtin_amdgcn_ballot_w64(odd) == 0u) return;
        static_assert(WAVES_K == 1, "a wave's columns are the tile's, which ends with a block and so within K");
        const uint8_t *const px = codes + (k0 + (lane & 15)) * BITS / 8;
        const float *const ps = scales + (k0 >> z.block_shift);
#pragma unroll 1
        for (int j = 0; j < FN; ++j) {
            const int64_t n = n0 + wn + j * 16 + (lane & 15);
            const T *const py = dy + min(n, z.N - 1);
            f32x4 plain[FK];
#pragma unroll
            for (int i = 0; i < FK; ++i) plain[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
            for (int64_t m = m0; m < m1; m += 4) {         // lane l holds row m + l / 16 of both; rows past the part's end count as zeros
                const int64_t row = min(m + (lane >> 4), m1 - 1);
                const bool in = m + (lane >> 4) < m1;
                const float step = ps[row * (z.K >> z.block_shift)], fy = in ? py[row * z.N] : 0.0f;
#pragma unroll
                for (int i = 0; i < FK; ++i) {
                    const uint32_t code = px[row * code_row + i * 16 * BITS / 8];
                    const float fx = in ? (float)code_field<BITS>(code, BITS == 8 ? 0 : lane & 1) * step : 0.0f;
                    plain[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(fx, fy, plain[i], 0, 0, 0);
                }
            }
            if (n >= z.N) continue;
#pragma unroll
            for (int i = 0; i < FK; ++i) {
                f32x4 *const at = reinterpret_cast<f32x4 *>(sums + n * z.K + k0 + i * 16 + (lane >> 4) * 4);     // its own store above
                f32x4 v = *at;
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = __builtin_fabsf(v[q]) < __builtin_inff() ? v[q] : plain[i][q];
                *at = v;
            }
        }
    }
}

// dw = the parts, added up in order; four elements a thread
template <typename T>
__global__ void __launch_bounds__(kThreads)
join_kernel(const float *__restrict__ parts, int count, int64_t vectors, T *__restrict__ dw, int64_t first)
{
    const int64_t i = first + (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= vectors) return;
    f32x4 sum = reinterpret_cast<const f32x4 *>(parts)[i];
    for (int p = 1; p < count; ++p) sum += reinterpret_cast<const f32x4 *>(parts)[p * vectors + i];
    if constexpr (sizeof(T) == 4) reinterpret_cast<f32x4 *>(dw)[i] = sum;
    else reinterpret_cast<u32x2 *>(dw)[i] = u32x2{bf16_narrow2(sum[0], sum[1]), bf16_narrow2(sum[2], sum[3])};
}

int32_t validate(int32_t dt, int64_t M, int64_t N, int64_t K)
{
    if (!dtype_ok(dt) || M < 0 || N < 0 || K < 0) return SLIMFIT_ERR_INVALID_ARG;
    if (N > (1 << 20) || K > (1 << 20) || M > ((int64_t)1 << 40)) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

template <typename T, int TN, int TK>
void launch_weight(const void *dy, const uint8_t *codes, const float *scales, int bits, const Sizes &z, const WeightPlan &plan, void *dw, float *parts, hipStream_t st)
{
    const unsigned grid = (unsigned)(plan.tiles * plan.splits);
    const T *y = static_cast<const T *>(dy);
    T *out = static_cast<T *>(dw);
    constexpr int E = 16 / sizeof(T);
    auto go = [&](auto b) {
        constexpr int BITS = decltype(b)::value;
        if (z.N % E == 0) {
            launch(weight_kernel<T, BITS, TN, TK, kAligned>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
        } else if constexpr (TN < 256) {                   // (tiles 256 wide are planned for aligned rows alone)
            if (z.N > E) launch(weight_kernel<T, BITS, TN, TK, kAnywhere>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
            else launch(weight_kernel<T, BITS, TN, TK, kShort>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
        }
    };
    if (bits == 8) go(std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 4>{});
}

}  // namespace
}  // namespace slimfit

using namespace slimfit;

extern "C" int32_t slimfit_weight_grad_dequant_workspace(int32_t dt, int32_t block, int64_t M, int64_t N, int64_t K, size_t *bytes)
{
    const int32_t rc = validate(dt, M, N, K);
    if (rc != SLIMFIT_OK) return rc;
    if (block != 32 && block != 64 && block != 128 && block != 256) return SLIMFIT_ERR_UNSUPPORTED;
    if (!bytes) return SLIMFIT_ERR_INVALID_ARG;
    *bytes = N == 0 || K == 0 ? 0 : WeightPlan(dt, block, M, N, K).workspace(N, K);
    return SLIMFIT_OK;
}

extern "C" int32_t slimfit_weight_grad_dequant(const void *dy, int32_t dt, const uint8_t *codes, const float *scales, int32_t bits, int32_t block,
                                               int64_t M, int64_t N, int64_t K, void *dw, void *workspace, size_t workspace_bytes, void *stream)
{
    StreamScope capture_aware(stream);
    int32_t rc = validate(dt, M, N, K);
    if (rc != SLIMFIT_OK) return rc;
    if ((bits != 4 && bits != 8) || (block != 32 && block != 64 && block != 128 && block != 256) || K % block != 0) return SLIMFIT_ERR_UNSUPPORTED;
    if (N == 0 || K == 0) return SLIMFIT_OK;
    if (!dw || (M > 0 && (!dy || !codes || !scales))) return SLIMFIT_ERR_INVALID_ARG;
    if (!aligned_to(dw, 16) || !aligned_to(dy, 16) || !aligned_to(codes, 16) || !aligned_to(scales, 16)) return SLIMFIT_ERR_ALIGNMENT;
    const size_t e = dtype_size(dt), out = (size_t)N * (size_t)K * e, in = (size_t)M * (size_t)N * e, kept = (size_t)M * (size_t)K;
    const size_t code_bytes = kept * (size_t)bits / 8, scale_bytes = kept / (size_t)block * 4;
    if (meet(dw, out, dy, in) || meet(dw, out, codes, code_bytes) || meet(dw, out, scales, scale_bytes)) return SLIMFIT_ERR_INVALID_ARG;
    const WeightPlan plan(dt, block, M, N, K);
    const size_t need = plan.workspace(N, K);
    if (plan.tiles > kMaxGridThreads / kThreads / plan.splits) return SLIMFIT_ERR_UNSUPPORTED;
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return SLIMFIT_ERR_WORKSPACE;
        if (!aligned_to(workspace, 16)) return SLIMFIT_ERR_ALIGNMENT;
        if ((rc = check_device_range(workspace, need)) != SLIMFIT_OK) return rc;
    }
    if ((rc = check_device_range(dw, out)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(dy, in)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(codes, code_bytes)) != SLIMFIT_OK) return rc;
    if ((rc = check_device_range(scales, scale_bytes)) != SLIMFIT_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Sizes z = {M, N, K, plan.split_rows, (int)tiles_of(N, plan.tile_n), (int)tiles_of(K, plan.tile_k), (int)plan.splits, __builtin_ctz((unsigned)block)};
    float *parts = need > 0 ? static_cast<float *>(workspace) : nullptr;
    if (dt == SLIMFIT_BF16 && plan.tile_n == 256) launch_weight<uint16_t, 256, 128>(dy, codes, scales, bits, z, plan, dw, parts, st);
    else if (dt == SLIMFIT_BF16) launch_weight<uint16_t, 128, 128>(dy, codes, scales, bits, z, plan, dw, parts, st);
    else if (plan.tile_k == 64) launch_weight<float, 128, 64>(dy, codes, scales, bits, z, plan, dw, parts, st);
    else launch_weight<float, 128, 32>(dy, codes, scales, bits, z, plan, dw, parts, st);
    if (parts) {
        const int64_t vectors = N * K / 4;
        constexpr int64_t kMost = kMaxGridThreads / kThreads * kThreads;
        for (int64_t first = 0; first < vectors; first += kMost) {
            const unsigned blocks = (unsigned)tiles_of(vectors - first < kMost ? vectors - first : kMost, kThreads);
            if (dt == SLIMFIT_BF16) launch(join_kernel<uint16_t>, blocks, kThreads, 0, st, parts, (int)plan.splits, vectors, static_cast<uint16_t *>(dw), first);
            else launch(join_kernel<float>, blocks, kThreads, 0, st, parts, (int)plan.splits, vectors, static_cast<float *>(dw), first);
        }
    }
    return launch_status();
}
