// Which launch a windowed prefill is: one tile a workgroup (window_tile.hip) or prefill.hip's.  Plain C++ (see
// prefill_deal.hpp): a host program can ask.
#pragma once

#include <algorithm>

#include "launch_grid.hpp"
#include "prefill_deal.hpp"
#include "window.hpp"

namespace coopt {

// Sets of 16 places that a tile of one wavefront can have: two where their sums and a group in flight fit the registers.
inline int window_tile_sets(const coopt_shape* sh) { return sh->head_dim == 128 && sh->kv_dtype == COOPT_KV_FP16 ? 1 : 2; }

constexpr int kWindowTileGroups = 64;       // two-block groups per wavefront: two registers of block numbers

// What a launch takes, in us, by a model of its two sides that was fitted to 250 measurements (dims 128 / 64; 11 % off
// on average, and what it chooses takes 1.7 % longer than the best choice, 22 % at most; it is off most often for fp16,
// whose views from the L2 it takes for slower than they are: of the rows below 30.8 us where 26.4 was to be had, 33.0
// where 30.1).  A tile's own time: for every group of a wavefront 0.68 / 0.56 (two sets: 1.12 / 0.74), or what one CU
// reads of its view (97 GB/s), and the merge.  The chip's: of a SIMD, 3 / 1.7 for a wavefront and 0.39 / 0.22 for its
// groups (two sets: 3.3 / 2 and 0.64 / 0.36), times the wavefronts that it has, half way to the next whole number; or
// the views from the L2 (21 TB/s) or the pairs' from HBM.  The longer one counts, and 0.39 of the other.
inline double tile_us(const coopt_shape* sh, double tiles, int groups, int waves, int sets)
{
    const bool wide = sh->head_dim == 128, two = sets == 2;
    const double group_bytes = 2.0 * sh->block_size * (sh->kv_dtype == COOPT_KV_FP16 ? 4.0 * sh->head_dim : 2.0 * sh->head_dim + 8);
    const double merge = waves == 1 ? 0.0 : waves == 2 ? 0.5 : 1.1;
    const double step = wide ? (two ? 1.12 : 0.68) : (two ? 0.74 : 0.56);
    const double own = std::max(step * ((groups + waves - 1) / waves) + merge, groups * group_bytes / 97e3);
    double on_simd = tiles * waves / 1024;
    if (on_simd > 1.0) on_simd = 0.5 * (on_simd + (double)(long long)(on_simd + 0.9999));
    const double of_wave = (wide ? (two ? 3.3 : 3.0) : (two ? 2.0 : 1.7)) + (wide ? (two ? 0.64 : 0.39) : (two ? 0.36 : 0.22)) * groups / waves;
    const double chip = std::max({on_simd * of_wave, tiles * groups * group_bytes / 21e6,
                                  (double)sh->num_seqs * sh->num_kv_heads * groups * group_bytes / 5.3e6});
    return 3.0 + std::max(own, chip) + 0.39 * std::min(own, chip);
}

// prefill.hip's launch: its plan's stages at 4 / 2.6 us (0.85 of it for fp16; 0.7 where a pair has 8 tiles at most), and the
// launch.  The plan takes every chunk for the longest; where rows are missing, what is left of its workgroups counts,
// of which every sequence has one per pair, and as they are not all as long, a round of them is not whole.
inline double stream_us(const coopt_shape* sh, long long rows, int max_chunk_len, long long tokens)
{
    const PrefillLaunchPlan plan(sh, max_chunk_len, true, tokens);
    const int G = sh->num_q_heads / sh->num_kv_heads;
    const double wgs = (double)sh->num_kv_heads * ((double)G * (double)rows / (16 * plan.wg_tiles) + sh->num_seqs);
    const double stages = (double)(tokens + (plan.wg_tiles + G - 1) / G * 16) / kPrefillStageTokens;
    const bool even = rows >= (long long)sh->num_seqs * max_chunk_len;
    const double rounds = even ? (double)(long long)(wgs / kPrefillCUs + 1.0) : std::max(1.0, wgs / kPrefillCUs);
    const double real = rounds * (2.3 + stages);
    return 3.0 + (sh->head_dim == 128 ? 4.0 : 2.6) * (plan.nr == 1 ? 0.7 : sh->kv_dtype == COOPT_KV_FP16 ? 0.85 : 1.0) *
                     std::min(plan.cost, real);
}

// Tiles of a launch: of every sequence as many as the longest chunk has, or what that many rows have, with a partly filled
// one per sequence.
inline long long window_tiles(const coopt_shape* sh, long long rows, int max_chunk_len, int places)
{
    const long long G = sh->num_q_heads / sh->num_kv_heads;
    const long long even = sh->num_seqs * ((max_chunk_len * G + places - 1) / places), found = rows * G / places + sh->num_seqs;
    return sh->num_kv_heads * (sh->num_seqs == 1 || rows >= (long long)sh->num_seqs * max_chunk_len ? even : found);
}

// In us, 128 dims unless said: tiles of 16 places with 1, 2 and 4 wavefronts, of 32 with one / prefill.hip:
//   40 heads over 8, E4M3     64 rows: window 64 7.0 6.0 6.4, 8.5 / 15.0   256 10.9 8.1 7.2, 14.4 / 18.8   1024 26.4 16.5 11.2, 37.6 / 23.2
//     1000 rows               16 14.6 20.0 29.2, 12.0 / 14.6   256 25.0 29.0 35.9, 23.2 / 22.9   1024 61.0 62.3 63.6, 59.2 / 41.9
//     4 x 512 rows            16 25.0 38.0 58.9, 20.6 / 27.5   128 32.5 40.4 68.5, 27.8 / 36.0   1024 99.5 114 127, 92.7 / 80.4
//     8 x 2000 rows           16 165 275 452, 116 / 130   128 219 291 527, 166 / 176   512 390 470 705, 302 / 267
//     512 rows and 63 x 1     256 20.0 26.0 32.1, 22.2 / 81.8   1024 51.3 61.5 64.7, 58.2 / 170
//   8 heads over 8, fp16      4 x 512 rows: 16 6.9 7.8 12.3 / 18.6, 512 18.1 17.3 22.0 / 32.3, 1024 30.1 31.9 33.0 / 36.2
//   64 dims, 32 over 8, E4M3  8 x 2000 rows: 16 70 120 195, 48 / 71   256 128 166 246, 101 / 135   1024 281 310 386, 235 / 235
//   64 dims, 32 over 8, fp16  64 rows: 1024 18.4 11.8 8.5, 26.5 / 15.9   1000 rows: 16 7.3 11.2 14.9, 6.7 / 9.4, 1024 26.4 31.8 30.3, 28 / 30.8
// Wavefronts per tile (1, 2 or 4; eight were no faster anywhere), or 0 where the launch is prefill.hip's, and the sets of
// 16 places (two for one wavefront only: several are for few tiles).  rows: of all sequences, or less than 0 where only
// the longest chunk is known -- as to a caller who asks for a workspace: where that already decides for tiles, there is
// none for anything else.
inline int window_tile_waves(const coopt_shape* sh, long long rows, int max_chunk_len, const Window& window, int* sets = nullptr)
{
    const long long all = (long long)sh->num_seqs * max_chunk_len;
    const bool known = rows >= 0 && rows < all;
    double best_us = stream_us(sh, known ? rows : all, max_chunk_len, window_row_tokens(sh, window));
    if (known && window_tile_waves(sh, -1, max_chunk_len, window) > 0) best_us = 1e30;
    int best = 0;
    for (int n = 1; n <= window_tile_sets(sh); ++n) {
        const int groups = (window_shape(sh, window, 16 * n).max_blocks_per_seq + 1) / 2;
        const long long tiles = window_tiles(sh, known ? rows : all, max_chunk_len, 16 * n);
        if (tiles > kMaxWorkgroups) continue;
        for (int waves = 1; waves <= (n > 1 ? 1 : 4); waves *= 2) {
            if ((groups + waves - 1) / waves > kWindowTileGroups) continue;
            const double us = tile_us(sh, (double)tiles, groups, waves, n);
            if (us < best_us) {
                best_us = us;
                best = waves;
                if (sets) *sets = n;
            }
        }
    }
    return best;
}

}  // namespace coopt
