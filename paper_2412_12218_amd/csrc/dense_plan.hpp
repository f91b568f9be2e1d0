// Which kernel, tile and how many parts of the contraction a product of the dense layer takes (linear.hip).  Plain C++, so that a host program can ask.
#pragma once
#include <math.h>
#include <stdint.h>

namespace ftc {

// Tiles of the result.
enum { DENSE_64 = 0, DENSE_128 = 1, DENSE_256 = 2 };
constexpr int dense_side(int tile) { return 64 << tile; }

struct DensePlan {
    int tile, splits, k_each;
};

inline int64_t dense_parts(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t dense_tiles(int M, int N, int tile) { return dense_parts(M, dense_side(tile)) * dense_parts(N, dense_side(tile)); }

// Tile and parts of the contraction by an estimate of the time.  A step (128 bytes of the contraction) of a workgroup takes `alone` where it
// has a compute unit to itself and `shared` for each of the workgroups of one that is full, `most` of them; parts cost the second kernel, and
// writing and reading them once.  us, from products of 8192^3 (1780 with tiles of 64 / 1080 of 128 / 900 of 256), 4096 x 1024 x 1024 (16 / 15 / 31
// for Z, 22 / 25 / 30 for dW at the best number of parts), 20 000 x 768 x 768 (40 / 34 / 30, 52 / 49 / 50) and 65 536 x 1024 x 4096
// (852 / 652 / 582, 1000 / 596 / 485), the last two with parts of up to 16 tried: more lose (4096 x 1024 x 1024, dW of 2 / 4 / 8 / 16 parts: 28 / 25 / 27 / 39).  fp32, tiles of 64 / 128:
// 16 384 x 2048 x 2048 1069 / 748, 1032 x 3696 x 2920 209 / 180, 2708 x 1432 x 128 21 (four parts) / 25 (six).
struct DenseCost {
    float alone, shared;
    int most;
};
inline DensePlan dense_plan(int M, int N, int K, bool f32, bool fast)
{
    static constexpr DenseCost cost[2][3] = {{{0.45f, 0.22f, 5}, {0.79f, 0.53f, 2}, {1.74f, 1.74f, 1}}, {{0.75f, 0.49f, 4}, {1.55f, 1.46f, 2}, {0.f, 0.f, 0}}};
    constexpr float JOIN_US = 5.f, PART_BYTES_US = 4e6f;
    DensePlan best = {DENSE_64, 1, 64};
    if (M < 1 || N < 1 || K < 1) return best;
    float least = INFINITY;
    const int step = f32 ? 32 : 64;
    for (int tile = DENSE_64; tile <= (fast && !f32 ? DENSE_256 : DENSE_128); ++tile) {
        const DenseCost &c = cost[f32][tile];
        const float alone = fast ? c.alone : 1.5f * c.alone;  // rows that are not whole pieces: through registers
        const int64_t tiles = dense_tiles(M, N, tile);
        for (int want = 1; want <= 64; want = want < 8 ? want + 1 : want + want / 4) {
            DensePlan p = {tile, 1, static_cast<int>(dense_parts(dense_parts(K, want), 64) * 64)};
            p.splits = static_cast<int>(dense_parts(K, p.k_each));
            if (p.splits != want) continue;
            const int64_t groups = tiles * p.splits, room = 256ll * c.most, full = groups / room, rest = groups % room;
            const auto each = [&](int64_t n) { return n * c.shared > alone ? n * c.shared : alone; };
            float us = dense_parts(p.k_each, step) * (full * each(c.most) + (rest ? each((rest + 255) / 256) : 0.f));
            if (p.splits > 1) us += JOIN_US + 8.f * p.splits * M * N / PART_BYTES_US;
            if (us < least) {
                least = us;
                best = p;
            }
            if (tiles * want >= 2048) break;  // more workgroups than the chip holds
        }
    }
    return best;
}

// Whether M rows take the kernels of linear_rows.hip, which read B once on the vector units (two rows at most where its rows lie across the contraction, four
// where they lie along it).  A workgroup has the whole contraction there, so long ones take tiles, whose contraction comes in parts; and where B is large what
// counts is the rate, which tiles of 16-bit numbers have more of.  us of these kernels / of tiles, from Python:
//   across, bf16, one row   1024 -> 4096 8.1 / 10.9  1024 -> 16 384 8.0 / 8.9  1024 -> 32 768 14.3 / 11.8  2048 -> 8192 14.5 / 11.0  4096 -> 1024 9.3 / 11.0
//                           4096 -> 2048 13.3 / 11.0  4096 -> 14 336 41.5 / 23.3  16 384 -> 512 37.9 / 11.5;  two rows 2048 -> 2048 9.0 / 11.0  4096 -> 1024 12.8 / 11.1
//   across, fp32, one row   4096 -> 2048 15.1 / 15.0  4096 -> 8192 26 / 39  8192 -> 1024 26 / 19  8192 -> 4096 31 / 39;  two rows 4096 -> 1024 13.8 / 13.2
//   along, bf16, one row    4096 <- 4096 9.8 / 12.5  4096 <- 8192 19.7 / 14.5  2048 <- 8192 9.8 / 12.8  1024 <- 16 384 15.8 / 12.9  16 384 <- 2048 16.8 / 15.3
//                four rows  4096 <- 4096 11.2 / 12.4  2048 <- 4096 10.7 / 12.5  2048 <- 8192 16.4 / 12.5  1024 <- 8192 15.3 / 12.8
//   1024 -> 4096, bf16, more rows: across four 10.4 / 10.7, eight 17.1 / 10.7, along eight 15.7 / 13.9
//   along, fp32, two rows   1024 <- 32 768 46 / 47;  four rows 1024 <- 8192 18.3 / 18.9  1024 <- 16 384 34 / 31  2048 <- 16 384 38 / 43  8192 <- 8192 51 / 73
inline bool dense_few_rows(int M, int N, int K, bool f32, bool across)
{
    const int64_t numbers = static_cast<int64_t>(N) * K;
    if (across) {
        if (M > 2) return false;
        return static_cast<int64_t>(K) * M <= 4096 ? f32 || numbers <= (1ll << 34) / K : f32 && N >= 4096;
    }
    if (M > 4) return false;
    return f32 ? M <= 2 || K <= 8192 || K <= 8ll * N : numbers <= 1ll << 24 && K <= (M <= 2 ? 8192 : 4096);
}

}  // namespace ftc
