// Which tile and how many parts of the contraction the products of a grouped dense layer take (grouped_linear.hip).  The host knows the rows and the groups, not
// the rows of a group.  Plain C++, so that a host program can ask.
#pragma once
#include "dense_plan.hpp"

namespace ftc {

// Tiles of DENSE_64 .. DENSE_256, and one of 32 rows by 128 columns for groups of few rows.
enum { GROUPED_THIN = 3 };
constexpr int grouped_rows(int tile) { return tile == GROUPED_THIN ? 32 : dense_side(tile); }
constexpr int grouped_columns(int tile) { return tile == GROUPED_THIN ? 128 : dense_side(tile); }
constexpr int grouped_threads(int tile) { return tile == DENSE_256 ? 512 : 256; }

// Groups begin anywhere, and tiles (or chunks, in the weight gradient) of `side` rows begin anew with each, so n rows in groups have at most this many, those of groups
// without rows, one each in the weight gradient, included.
inline int64_t grouped_most(int n, int groups, int side) { return static_cast<int64_t>(n / side) + groups; }
// What a tile of a group leaves for a later kernel has a place by its number: group g, rows s .. e - 1, has the numbers from s / side + g on.  ceil((e - s) / side) <= e / side - s / side + 1,
// so the next group's are behind them, whatever the groups are, and all are below grouped_most().

// Tiles that n rows in groups come to, as far as the host can tell: a group's last one is half full, or less, where there are many groups of few rows.
inline int64_t grouped_tiles(int n, int groups, int N, int tile)
{
    const int used = groups < n ? groups : n;
    return (n / grouped_rows(tile) + (3ll * used + 4) / 5) * dense_parts(N, grouped_columns(tile));
}
// Whether tiles of 256 behind the last full turn of the compute units are taken in parts (grouped_kernel.hpp): where a second kernel for them is no waste, as it is launched
// before it is known how many tiles there are (5 us of 170 in a training step of 20 000 x 768 -> 768, whose 249 tiles are less than one turn).
constexpr int TAIL_LEAST = 256;  // indices of a part at least
inline bool grouped_tail_on(int n, int groups, int N, int K) { return K >= 2 * TAIL_LEAST && grouped_tiles(n, groups, N, DENSE_256) > 264; }

// Tiles of 256 have a compute unit each, so those behind the last 256 of a launch would take as long as 256 do.  Where these are at most half of 256 their contraction is taken
// in parts, for as many workgroups as there are units: each writes its part of a tile, and grouped_tail_kernel (grouped_kernel.hpp) adds them up.  us of 48 000 rows in 16 groups, 4096 -> 1024 in fp16, 776 tiles:
// 482 without, 440.
struct GroupedTail {
    int full, rest, parts;  // tiles in front, tiles in parts, parts of each
};
constexpr int TAIL_PARTS = 8;  // at most
constexpr GroupedTail grouped_tail(int64_t tiles, int K)
{
    const int rest = static_cast<int>(tiles % 256), full = static_cast<int>(tiles - rest);
    if (full == 0 || rest == 0 || rest > 128) return {static_cast<int>(tiles), 0, 1};
    const int fill = 256 / rest, most = K / TAIL_LEAST, parts = fill < TAIL_PARTS ? fill : TAIL_PARTS, take = parts < most ? parts : most;
    if (take < 2) return {static_cast<int>(tiles), 0, 1};
    return {full, rest, take};
}
// Indices of a part, whole steps; the last parts can be without any.
constexpr int tail_each(int K, int parts) { return ((K + parts - 1) / parts + 63) / 64 * 64; }

// Z and dX: n rows in groups.  As dense_plan() has it, with the tile of 32 rows at the cost of one of 64: it is as fast at reading weights and has half as many rows to be without.
// us of tiles of 64 / of 32 rows, 64 groups, 1024 -> 4096: 24 rows bf16 25 / 24, fp32 81 / 50; 200 rows 77 / 75, 207 / 135; 1000 rows 97 / 91, 248 / 172; larger tiles, other sizes: 8 rows in 8 groups,
// 4096 -> 512 in bf16 31 (64), 14 (64, in parts, as taken), 48 000 in 16, 4096 -> 1024 in fp16 706 (64), 482 (128), 440 (256); 20 000 in 8, 768 -> 768 50, 44 to 46, 49.
inline DensePlan grouped_plan(int n, int groups, int N, int K, bool f32, bool fast)
{
    static constexpr DenseCost cost[2][4] = {{{0.45f, 0.22f, 5}, {0.79f, 0.53f, 2}, {1.74f, 1.74f, 1}, {0.45f, 0.22f, 4}},
                                             {{0.75f, 0.49f, 4}, {1.55f, 1.46f, 2}, {0.f, 0.f, 0}, {0.75f, 0.49f, 4}}};
    constexpr float JOIN_US = 5.f, PART_BYTES_US = 4e6f, TAIL_US = 25.f;  // TAIL_US: the tiles of a last turn in parts (grouped_kernel.hpp)
    DensePlan best = {DENSE_64, 1, 64};
    if (n < 1 || groups < 1 || N < 1 || K < 1) return best;
    float least = INFINITY;
    const int step = f32 ? 32 : 64;
    for (int tile = DENSE_64; tile <= GROUPED_THIN; ++tile) {
        if (tile == DENSE_256 && (!fast || f32)) continue;
        const DenseCost &c = cost[f32][tile];
        const float alone = fast ? c.alone : 1.5f * c.alone;
        const int64_t tiles = grouped_tiles(n, groups, N, tile);
        const bool tail = tile == DENSE_256 && grouped_tail_on(n, groups, N, K);
        for (int want = 1; want <= 64; want = want < 8 ? want + 1 : want + want / 4) {
            DensePlan p = {tile, 1, static_cast<int>(dense_parts(dense_parts(K, want), 64) * 64)};
            p.splits = static_cast<int>(dense_parts(K, p.k_each));
            if (p.splits != want) continue;
            // how many tiles there are is known so well only, so nothing is made of how the last turn is filled
            const int64_t blocks = tiles * p.splits, share = (blocks + 255) / 256;
            const float steps = static_cast<float>(dense_parts(p.k_each, step));
            float us = steps * (share * c.shared > alone ? share * c.shared : alone);
            if (blocks > 256ll * c.most) us = tail && p.splits == 1 ? steps * alone * blocks / 256 + TAIL_US : steps * (c.shared * blocks / 256 + 0.5f * alone);
            if (p.splits > 1) us += JOIN_US + 8.f * p.splits * n * N / PART_BYTES_US;
            if (us < least) {
                least = us;
                best = p;
            }
            if (tiles * want >= 2048) break;
        }
    }
    return best;
}

// dW: a group's contraction is over its rows, in chunks of at most k_each of them, each for a workgroup a tile.  Time by the work of a compute unit, with half a chunk more a
// group, or by that of the longest chunk, whichever is more; parts are written and read once, those of groups of several chunks.
inline DensePlan grouped_dw_plan(int n, int groups, int M, int N, bool f32, bool fast)
{
    static constexpr DenseCost cost[2][3] = {{{0.45f, 0.22f, 5}, {0.79f, 0.53f, 2}, {1.74f, 1.74f, 1}}, {{0.75f, 0.49f, 4}, {1.55f, 1.46f, 2}, {0.f, 0.f, 0}}};
    constexpr float JOIN_US = 5.f, PART_BYTES_US = 4e6f;
    DensePlan best = {DENSE_64, 1, 64};
    if (n < 1 || groups < 1 || M < 1 || N < 1) return best;
    float least = INFINITY;
    const int step = f32 ? 32 : 64, used = groups < n ? groups : n;
    for (int tile = DENSE_64; tile <= (fast && !f32 ? DENSE_256 : DENSE_128); ++tile) {
        const DenseCost &c = cost[f32][tile];
        const float alone = fast ? c.alone : 1.5f * c.alone;
        const float tiles = static_cast<float>(dense_tiles(M, N, tile));
        for (int64_t want = 1; want <= 256; want = want < 8 ? want + 1 : want + want / 4) {
            DensePlan p = {tile, 1, static_cast<int>(dense_parts(dense_parts(n, want), 64) * 64)};
            p.splits = static_cast<int>(dense_parts(n, p.k_each));
            if (p.splits > 1 && 8.f * p.splits * M * N > 2e9f) break;  // parts of 2 GB
            const float rows = n + 0.5f * step * used, work = tiles * rows / step * c.shared / 256, longest = static_cast<float>(p.k_each) / step * alone;
            float us = work > longest ? work + 0.5f * longest : longest + 0.5f * work;
            if (p.splits > 1) us += JOIN_US + 8.f * p.splits * M * N / PART_BYTES_US;
            if (us < least) {
                least = us;
                best = p;
            }
        }
    }
    return best;
}
// Parts of a weight gradient: a group of several chunks, so of more than k_each rows, has those from 2 (s / k_each) on.  With q = e / k_each - s / k_each >= 1 it has at
// most q + 1 <= 2 q chunks, so the next group's are behind them.
inline int64_t grouped_dw_parts(int n, const DensePlan &p) { return p.k_each < n ? 2ll * (n / p.k_each) : 0; }

}  // namespace ftc
