// Tiles and parts of the weight gradients from the cache (weight_grad.hip); host code alone.
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>

#include "slimfit.h"

namespace slimfit {
namespace {

constexpr int kStep = 32;                                  // rows of the sum that a workgroup takes at a time

inline int64_t tiles_of(int64_t n, int tile) { return (n + tile - 1) / tile; }

// How wide the tiles are and among how many workgroups a tile's sum is shared: what takes the least time by this count of
// microseconds, measured over 20 sizes from 300 x 300 x 256 to 16384 x 4096 x 1024.  A step of 32 rows takes a + b * (workgroups on
// the fullest compute unit), of which `most` go on one at a time; rows of dy that begin anywhere cost `ragged` as much.  Parts are
// written and read again at 4.2 TB/s by a launch of 3 us.  (Chosen: 16384 x 4096 x 1024 bf16 256 wide in 4 parts 165 us, 128 wide in 3
// 187, in one 322; 4096 x 768 x 768 128 wide in 6 25, in one 72; 12608 x 1024 x 4096 fp32 in 2 403, in one 461; in 4, which the count
// puts at 433 against 415, 391.)
struct Pace {
    int tile_n, most;
    float a, b, ragged;
};
constexpr Pace kNarrow = {128, 4, 0.40f, 0.23f, 1.25f}, kSplit = {128, 4, 0.45f, 0.39f, 1.25f};
constexpr Pace kWide = {256, 2, 0.39f, 0.39f, 0.0f};       // for rows of dy that begin on 16 bytes alone: others cost 1.6 times as much and never gain

// The parts' memory is at most 256 MiB, a thousandth of the card's, or the size of x^, which this way of forming the product saves.
// (16384 x 6144 x 4096 bf16 in 2 parts of 201 MB 838 us, in one 943; 16384 x 5120 x 5120 945 in 3 of 315 MB, 950 in one;
// 36390 x 6579 x 1920 1191 in 6 of 303 MB, 1270 in 2 of 101.)
constexpr int64_t kPartsBytes = (int64_t)1 << 28;

struct WeightPlan {
    int tile_n, tile_k;
    int64_t tiles, splits, split_rows;
    WeightPlan(int32_t dt, int32_t block, int64_t M, int64_t N, int64_t K)
    {
        tile_k = dt == SLIMFIT_BF16 ? 128 : block >= 64 ? 64 : 32;
        const int64_t steps = tiles_of(M, kStep), saved = M * K * (dt == SLIMFIT_BF16 ? 2 : 4), most = saved > kPartsBytes ? saved : kPartsBytes;
        const bool ragged = N % (dt == SLIMFIT_BF16 ? 8 : 4) != 0;
        float best = 0.0f;
        auto look = [&](const Pace &p, int s) {
            const int64_t t = tiles_of(N, p.tile_n) * tiles_of(K, tile_k), full = 256 * p.most, groups = t * s, rest = groups % full;
            const float step = (float)(groups / full) * (p.a + p.b * (float)p.most) + (rest ? p.a + p.b * (float)tiles_of(rest, 256) : 0.0f);
            const float join = s > 1 ? 3.0f + (float)s * (float)N * (float)K * (8.0f / 4.2e6f) : 0.0f;
            const float time = (float)tiles_of(steps, s) * step * (ragged ? p.ragged : 1.0f) + join;
            if (best == 0.0f || time < best) {
                best = time;
                tile_n = p.tile_n;
                tiles = t;
                splits = s;
            }
        };
        tile_n = 128;
        tiles = splits = 1;
        for (const int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (s > 1 && (steps < 2 * s || s * N * K * 4 > most)) break;
            look(dt == SLIMFIT_BF16 ? kNarrow : kSplit, s);
            if (dt == SLIMFIT_BF16 && !ragged) look(kWide, s);
        }
        split_rows = tiles_of(steps, splits) * kStep;
        if (split_rows == 0) split_rows = kStep;
    }
    size_t workspace(int64_t N, int64_t K) const { return splits > 1 ? (size_t)splits * (size_t)N * (size_t)K * 4 : 0; }
};

}  // namespace
}  // namespace slimfit
