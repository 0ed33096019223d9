// Weight gradient of an active linear layer straight from the low-bit cache of its input (Alg. 4's dW = dY^T X with X as the
// cache gives it back): dw[n][k] = sum over m of dy[m][n] code[m][k] scale[m][k / block].
//
// Both operands lie across the sum: eight rows m of two columns are read as words, turned in registers and written to LDS as
// runs along m, which is what a lane hands to v_mfma_f32_16x16x32_bf16.  The codes become bf16 on that way.
//   bf16  x^ = code * scale rounded to bf16, as the cache gives it to a bf16 tensor.
//   fp32  the scale goes onto dy (a tile lies in one block), whose product is rounded to fp32 once and taken apart exactly
//         into three bf16 numbers; the codes are whole numbers that bf16 holds.  Three products in place of the six that two
//         fp32 operands take.
// Rows past M are read as zeros by the bounds of the buffer descriptors, which move along with the steps.  Where there are
// fewer tiles than the compute units can hold, the rows are shared out and the parts added up in order by a second kernel.
#include "common.hpp"

namespace slimfit {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kTileN = 128;

typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_of(const void *at, int64_t bytes)      // bytes from `at` to the matrix's end; reads past it give 0
{
    const int64_t most = 0xFFFFFFF0LL, n = bytes < 0 ? 0 : bytes < most ? bytes : most;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, (int)(uint32_t)n, 0x00020000);
}

// code c of BITS bits in byte (or nibble) i of a word whose fields have 2^(BITS-1) added: (field - 2^(BITS-1)) * step, exact but
// for the product's one rounding
template <int BITS>
__device__ __forceinline__ float field(uint32_t word, int i)
{
    return (float)((word >> (i * BITS)) & ((1u << BITS) - 1));
}

template <typename T, int TK> struct Config;
template <> struct Config<uint16_t, 128> { static constexpr int STEP = 64, PARTS = 1, KW = 4, MW = 8; };
template <> struct Config<float, 64> { static constexpr int STEP = 32, PARTS = 3, KW = 2, MW = 4; };
template <> struct Config<float, 32> { static constexpr int STEP = 32, PARTS = 3, KW = 2, MW = 2; };

template <int ROW_BYTES>
__device__ __forceinline__ int chunk_at(int row, int chunk)
{
    return row * ROW_BYTES + ((chunk ^ ((row >> 1) & (ROW_BYTES / 16 - 1))) << 4);
}

struct Sizes {
    int64_t M, N, K, split_rows;           // split_rows: rows of a part, a multiple of the step
    int tiles_n, tiles_k, block_shift;
};

template <typename T, int BITS, int TK, bool ODD>
__global__ void __launch_bounds__(kThreads)
weight_kernel(const T *__restrict__ dy, const uint8_t *__restrict__ codes, const float *__restrict__ scales, T *__restrict__ dw,
              float *__restrict__ parts, Sizes z)
{
    using C = Config<T, TK>;
    constexpr int STEP = C::STEP, PARTS = C::PARTS, KW = C::KW, MW = C::MW, ROW = STEP * 2, CHUNKS = STEP / 8;
    constexpr bool WIDE = sizeof(T) == 4;
    constexpr int CA = CHUNKS / 4;                         // runs of eight rows of dy a thread
    constexpr int FN = kTileN / 2 / 16, FK = TK / 2 / 16;
    constexpr int PART = kTileN * ROW;
    __shared__ __align__(16) char lds[PARTS * PART + TK * ROW];
    const int t = threadIdx.x, lane = t & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int tiles = z.tiles_n * z.tiles_k;
    const int per = tiles / 8, b0 = (int)blockIdx.x, id = b0 < per * 8 ? (b0 % 8) * per + b0 / 8 : b0;
    const int band = id / (4 * z.tiles_k), in_band = id % (4 * z.tiles_k), height = min(4, z.tiles_n - 4 * band);
    const int64_t n0 = (int64_t)(band * 4 + in_band % height) * kTileN, k0 = (int64_t)(in_band / height) * TK;
    const int64_t m0 = (int64_t)blockIdx.y * z.split_rows, m1 = min(m0 + z.split_rows, z.M);
    const int steps = (int)((m1 - m0 + STEP - 1) / STEP);

    const int64_t dy_row = z.N * (int64_t)sizeof(T), code_row = z.K * BITS / 8, scale_row = (z.K >> z.block_shift) * 4;
    int at_dy[CA][8], at_code[MW], at_scale[WIDE ? 8 * CA : MW];
#pragma unroll
    for (int q = 0; q < CA; ++q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) at_dy[q][i] = (int)(((wave * CA + q) * 8 + i) * dy_row + (n0 + 2 * lane) * (int64_t)sizeof(T));
    }
    constexpr int ACROSS = TK / KW;
    const int kx = t % ACROSS * KW, mx = t / ACROSS * MW;  // the thread's codes of the tile
    static_assert(kThreads / ACROSS * MW == STEP, "the codes of a step");
#pragma unroll
    for (int i = 0; i < MW; ++i) at_code[i] = (int)((mx + i) * code_row + (k0 + kx) * BITS / 8);
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < 8 * CA; ++i) at_scale[i] = (int)((wave * CA * 8 + i) * scale_row + (k0 >> z.block_shift) * 4);
    } else {
#pragma unroll
        for (int i = 0; i < MW; ++i) at_scale[i] = (int)((mx + i) * scale_row + ((k0 + kx) >> z.block_shift) * 4);
    }

    uint32_t hy[CA][8][WIDE ? 2 : 1], hc[MW];
    float hs[WIDE ? 8 * CA : MW];
    auto load = [&](int64_t m) {
        const Buffer by = buffer_of(reinterpret_cast<const char *>(dy) + m * dy_row, (z.M - m) * dy_row);
        const Buffer bc = buffer_of(codes + m * code_row, (z.M - m) * code_row);
        const Buffer bs = buffer_of(reinterpret_cast<const char *>(scales) + m * scale_row, (z.M - m) * scale_row);
#pragma unroll
        for (int q = 0; q < CA; ++q) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (WIDE) {
                    if constexpr (ODD) {
                        hy[q][i][0] = __builtin_amdgcn_raw_buffer_load_b32(by, at_dy[q][i], 0, 0);
                        hy[q][i][1] = __builtin_amdgcn_raw_buffer_load_b32(by, at_dy[q][i] + 4, 0, 0);
                    } else {
                        const auto v = __builtin_amdgcn_raw_buffer_load_b64(by, at_dy[q][i], 0, 0);
                        hy[q][i][0] = v[0];
                        hy[q][i][1] = v[1];
                    }
                } else if constexpr (ODD) {
                    hy[q][i][0] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(by, at_dy[q][i], 0, 0) |
                                  (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(by, at_dy[q][i] + 2, 0, 0) << 16;
                } else {
                    hy[q][i][0] = __builtin_amdgcn_raw_buffer_load_b32(by, at_dy[q][i], 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < MW; ++i) {
            constexpr int BYTES = KW * BITS;               // in bits
            if constexpr (BYTES == 32) hc[i] = __builtin_amdgcn_raw_buffer_load_b32(bc, at_code[i], 0, 0);
            else if constexpr (BYTES == 16) hc[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(bc, at_code[i], 0, 0);
            else hc[i] = (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(bc, at_code[i], 0, 0);
        }
#pragma unroll
        for (int i = 0; i < (WIDE ? 8 * CA : MW); ++i) hs[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(bs, at_scale[i], 0, 0));
    };
    auto store = [&]() {
#pragma unroll
        for (int q = 0; q < CA; ++q) {
            const int chunk = wave * CA + q;
            if constexpr (WIDE) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {              // columns 2 lane and 2 lane + 1
                    uint32_t h[4], m[4], l[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float a = __builtin_bit_cast(float, hy[q][2 * i][c]) * hs[q * 8 + 2 * i];
                        float b = __builtin_bit_cast(float, hy[q][2 * i + 1][c]) * hs[q * 8 + 2 * i + 1];
                        h[i] = bf16_narrow2(a, b);
                        a -= __builtin_bit_cast(float, h[i] << 16);
                        b -= __builtin_bit_cast(float, h[i] & 0xFFFF0000u);
                        m[i] = bf16_narrow2(a, b);
                        a -= __builtin_bit_cast(float, m[i] << 16);
                        b -= __builtin_bit_cast(float, m[i] & 0xFFFF0000u);
                        l[i] = bf16_narrow2(a, b);
                    }
                    char *to = lds + chunk_at<ROW>(2 * lane + c, chunk);
                    *reinterpret_cast<u32x4 *>(to) = u32x4{h[0], h[1], h[2], h[3]};
                    *reinterpret_cast<u32x4 *>(to + PART) = u32x4{m[0], m[1], m[2], m[3]};
                    *reinterpret_cast<u32x4 *>(to + 2 * PART) = u32x4{l[0], l[1], l[2], l[3]};
                }
            } else {
                uint32_t even[4], odd[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    even[i] = __builtin_amdgcn_perm(hy[q][2 * i + 1][0], hy[q][2 * i][0], 0x05040100u);
                    odd[i] = __builtin_amdgcn_perm(hy[q][2 * i + 1][0], hy[q][2 * i][0], 0x07060302u);
                }
                *reinterpret_cast<u32x4 *>(lds + chunk_at<ROW>(2 * lane, chunk)) = u32x4{even[0], even[1], even[2], even[3]};
                *reinterpret_cast<u32x4 *>(lds + chunk_at<ROW>(2 * lane + 1, chunk)) = u32x4{odd[0], odd[1], odd[2], odd[3]};
            }
        }
        constexpr uint32_t kFlip = BITS == 8 ? 0x80808080u : 0x88888888u;
        constexpr float kBias = BITS == 8 ? 128.0f : 8.0f;
#pragma unroll
        for (int c = 0; c < KW; ++c) {
            uint32_t x[MW / 2];
#pragma unroll
            for (int i = 0; i < MW; i += 2) {
                float a = field<BITS>(hc[i] ^ kFlip, c), b = field<BITS>(hc[i + 1] ^ kFlip, c);
                if constexpr (WIDE) {
                    a -= kBias;
                    b -= kBias;
                } else {                                   // (field - bias) * scale, rounded once: bias * scale is exact
                    a = fmaf(a, hs[i], -kBias * hs[i]);
                    b = fmaf(b, hs[i + 1], -kBias * hs[i + 1]);
                }
                x[i / 2] = bf16_narrow2(a, b);
            }
            char *to = lds + PARTS * PART + chunk_at<ROW>(kx + c, mx / 8) + mx % 8 * 2;
            if constexpr (MW == 8) *reinterpret_cast<u32x4 *>(to) = u32x4{x[0], x[1], x[2], x[3]};
            else if constexpr (MW == 4) *reinterpret_cast<u32x2 *>(to) = u32x2{x[0], x[1]};
            else *reinterpret_cast<uint32_t *>(to) = x[0];
        }
    };

    f32x4 acc[FK][FN];
#pragma unroll
    for (int i = 0; i < FK; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int wn = (wave >> 1) * (kTileN / 2), wk = (wave & 1) * (TK / 2);
    load(m0);
    for (int s = 0; s < steps; ++s) {
        store();
        load(m0 + (int64_t)(s + 1) * STEP);                // past the last step: the next part's rows, or none
        __syncthreads();
#pragma unroll
        for (int h = 0; h < STEP / 32; ++h) {
            bf16x8 fx[FK];
#pragma unroll
            for (int i = 0; i < FK; ++i)
                fx[i] = *reinterpret_cast<const bf16x8 *>(lds + PARTS * PART + chunk_at<ROW>(wk + i * 16 + (lane & 15), h * 4 + (lane >> 4)));
#pragma unroll
            for (int j = 0; j < FN; ++j) {
#pragma unroll
                for (int p = PARTS - 1; p >= 0; --p) {     // small parts first
                    const bf16x8 fy = *reinterpret_cast<const bf16x8 *>(lds + p * PART + chunk_at<ROW>(wn + j * 16 + (lane & 15), h * 4 + (lane >> 4)));
#pragma unroll
                    for (int i = 0; i < FK; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[i], fy, acc[i][j], 0, 0, 0);
                }
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int64_t n = n0 + wn + j * 16 + (lane & 15);
        if (n >= z.N) continue;
#pragma unroll
        for (int i = 0; i < FK; ++i) {
            const int64_t k = k0 + wk + i * 16 + (lane >> 4) * 4;
            if (k >= z.K) continue;
            const f32x4 v = acc[i][j];
            if (parts) *reinterpret_cast<f32x4 *>(parts + (int64_t)blockIdx.y * z.N * z.K + n * z.K + k) = v;
            else if constexpr (WIDE) *reinterpret_cast<f32x4 *>(dw + n * z.K + k) = v;
            else *reinterpret_cast<u32x2 *>(dw + n * z.K + k) = u32x2{bf16_narrow2(v[0], v[1]), bf16_narrow2(v[2], v[3])};
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

int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }

struct Plan {
    int tile_k, step;
    int64_t tiles, splits, split_rows;
    Plan(int32_t dt, int32_t block, int64_t M, int64_t N, int64_t K)
    {
        tile_k = dt == SLIMFIT_BF16 ? 128 : block >= 64 ? 64 : 32;
        step = dt == SLIMFIT_BF16 ? 64 : 32;
        tiles = tiles_of(N, kTileN) * tiles_of(K, tile_k);
        const int64_t steps = M / step + 1;
        splits = 1;
        while (splits < 32 && tiles * splits * 2 <= 768 && steps >= splits * 2 * 4) splits *= 2;
        split_rows = tiles_of(tiles_of(M, (int)splits), step) * step;
        if (split_rows == 0) split_rows = step;
    }
    size_t workspace(int64_t N, int64_t K) const { return splits > 1 ? (size_t)splits * (size_t)N * (size_t)K * 4 : 0; }
};

int32_t validate(int32_t dt, int64_t M, int64_t N, int64_t K)
{
    if (!dtype_ok(dt) || M < 0 || N < 0 || K < 0) return SLIMFIT_ERR_INVALID_ARG;
    if (N > (1 << 20) || K > (1 << 20) || M > ((int64_t)1 << 40)) return SLIMFIT_ERR_UNSUPPORTED;
    return SLIMFIT_OK;
}

template <typename T, int TK>
void launch_weight(const void *dy, const uint8_t *codes, const float *scales, int bits, const Sizes &z, const Plan &plan, void *dw, float *parts, hipStream_t st)
{
    const dim3 grid((unsigned)plan.tiles, (unsigned)plan.splits);
    const T *y = static_cast<const T *>(dy);
    T *out = static_cast<T *>(dw);
    const bool odd = z.N % 2 != 0;
    if (bits == 8) {
        if (odd) launch(weight_kernel<T, 8, TK, true>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
        else launch(weight_kernel<T, 8, TK, false>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
    } else {
        if (odd) launch(weight_kernel<T, 4, TK, true>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
        else launch(weight_kernel<T, 4, TK, false>, grid, kThreads, 0, st, y, codes, scales, out, parts, z);
    }
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
    *bytes = N == 0 || K == 0 ? 0 : Plan(dt, block, M, N, K).workspace(N, K);
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
    const Plan plan(dt, block, M, N, K);
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
    const Sizes z = {M, N, K, plan.split_rows, (int)tiles_of(N, kTileN), (int)tiles_of(K, plan.tile_k), __builtin_ctz((unsigned)block)};
    float *parts = need > 0 ? static_cast<float *>(workspace) : nullptr;
    if (dt == SLIMFIT_BF16) launch_weight<uint16_t, 128>(dy, codes, scales, bits, z, plan, dw, parts, st);
    else if (plan.tile_k == 64) launch_weight<float, 64>(dy, codes, scales, bits, z, plan, dw, parts, st);
    else launch_weight<float, 32>(dy, codes, scales, bits, z, plan, dw, parts, st);
    if (parts) {
        const int64_t vectors = N * K / 4;
        const unsigned blocks = (unsigned)((vectors + kThreads - 1) / kThreads);
        if (dt == SLIMFIT_BF16) launch(join_kernel<uint16_t>, blocks, kThreads, 0, st, parts, (int)plan.splits, vectors, static_cast<uint16_t *>(dw), 0);
        else launch(join_kernel<float>, blocks, kThreads, 0, st, parts, (int)plan.splits, vectors, static_cast<float *>(dw), 0);
    }
    return launch_status();
}
