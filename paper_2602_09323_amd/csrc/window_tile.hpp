// Which launch a windowed prefill is: one tile a workgroup (window_tile.hip) or prefill.hip's.  Plain C++ (see
// prefill_deal.hpp): a host program can ask.
#pragma once

#include <algorithm>

#include "launch_grid.hpp"
#include "prefill_deal.hpp"
#include "window.hpp"

namespace coopt {

constexpr int kWindowTileGroups = 64;       // two-block groups per wavefront: two registers of block numbers

// What a launch takes, in us, by a model of its two sides that measurements gave (dims 128 / 64).  A tile's own time: 4.2
// and 0.6 for every group of a wavefront, or what one CU reads of its view (64 GB/s), and the merge.  The chip's: of a
// SIMD, 3 / 2 for a wavefront and 0.39 / 0.26 for a group, or the views from the L2 (15 TB/s) or the pairs' from HBM.
// The longer one counts, and 0.4 of the other.
inline double tile_us(const coopt_shape* sh, double tiles, int groups, int waves)
{
    const double group_bytes = 2.0 * sh->block_size * (sh->kv_dtype == COOPT_KV_FP16 ? 4.0 * sh->head_dim : 2.0 * sh->head_dim + 8);
    const double merge = waves == 1 ? 0.0 : waves == 2 ? 0.4 : 1.0;
    const double own = std::max(0.6 * ((groups + waves - 1) / waves) + merge, groups * group_bytes / 64e3);
    const double chip = std::max({tiles * (3.0 * waves + 0.39 * groups) / 1024 * (sh->head_dim == 128 ? 1.0 : 0.65),
                                  tiles * groups * group_bytes / 15e6, (double)sh->num_seqs * sh->num_kv_heads * groups * group_bytes / 5.3e6});
    return 4.2 + std::max(own, chip) + 0.4 * std::min(own, chip);
}

// prefill.hip's launch: its plan's stages at 4 / 2.6 us (0.7 of it where a pair has 8 tiles at most), and the launch.  The
// plan takes every chunk for the longest; where rows are missing, what is left of its workgroups counts, of which
// every sequence has one per pair.
inline double stream_us(const coopt_shape* sh, long long rows, int max_chunk_len, long long tokens)
{
    const PrefillLaunchPlan plan(sh, max_chunk_len, true, tokens);
    const int G = sh->num_q_heads / sh->num_kv_heads;
    const double wgs = (double)sh->num_kv_heads * ((double)G * (double)rows / (16 * plan.wg_tiles) + sh->num_seqs);
    const double stages = (double)(tokens + (plan.wg_tiles + G - 1) / G * 16) / kPrefillStageTokens;
    const double real = (double)(long long)(wgs / kPrefillCUs + 1.0) * (2.3 + stages);
    return 3.0 + (sh->head_dim == 128 ? 4.0 : 2.6) * (plan.nr == 1 ? 0.7 : 1.0) * std::min(plan.cost, real);
}

// Tiles of 16 places of a launch: of every sequence as many as the longest chunk has, or what that many rows have,
// with a partly filled one per sequence.
inline long long window_tiles(const coopt_shape* sh, long long rows, int max_chunk_len)
{
    const long long G = sh->num_q_heads / sh->num_kv_heads;
    const long long even = sh->num_seqs * ((max_chunk_len * G + 15) / 16), found = rows * G / 16 + sh->num_seqs;
    return sh->num_kv_heads * (sh->num_seqs == 1 || rows >= (long long)sh->num_seqs * max_chunk_len ? even : found);
}

// In us, 128 dims unless said, tiles (wavefronts a tile) / prefill.hip:
//   40 heads over 8, E4M3     64 rows: window 64 6.0 (2) / 15.0, 256 7.2 (4) / 18.7, 1024 11.4 (4) / 23.1, 4096 28.5 (4) / 32.7
//     256 rows                64 7.8 (1) / 15.3, 1024 24.8 (2) / 31.6
//     1000 rows               16 14.7 (1) / 14.7, 256 26.9 (1) / 23.0, 1024 61.6 (2) / 42.2
//     4 x 512 rows            16 24.1 (1) / 26.5, 128 32.8 (1) / 36.0, 256 46.4 (1) / 43.9
//     512 rows and 63 x 1     256 19.5 / 82.9, 1024 57.1 / 172.2, 4096 200 / 519
//   8 heads over 8, fp16      4 x 512 rows: 16 7.0 (1) / 18.5, 512 22.4 (2) / 32.6, 1024 35.9 / 36.8
//   64 dims, 32 over 8, fp16  64 rows: 1024 8.4 (4) / 15.6   1000 rows: 16 7.4 (1) / 9.3, 512 17.4 (1) / 20.5, 1024 30.9 (4) / 31.5
// Wavefronts per tile (1, 2 or 4; eight were no faster anywhere), or 0 where the launch is prefill.hip's.  rows: of all
// sequences, or less than 0 where only the longest chunk is known -- as to a caller who asks for a workspace: where
// that already decides for tiles, there is none for anything else.
inline int window_tile_waves(const coopt_shape* sh, long long rows, int max_chunk_len, const Window& window)
{
    const long long all = (long long)sh->num_seqs * max_chunk_len;
    const bool known = rows >= 0 && rows < all;
    const int groups = (window_shape(sh, window, 16).max_blocks_per_seq + 1) / 2;
    const long long tiles = window_tiles(sh, known ? rows : all, max_chunk_len);
    if (tiles > kMaxWorkgroups) return 0;
    double best_us = stream_us(sh, known ? rows : all, max_chunk_len, window_row_tokens(sh, window));
    if (known && window_tile_waves(sh, -1, max_chunk_len, window) > 0) best_us = 1e30;
    int best = 0;
    for (int waves = 1; waves <= 4; waves *= 2) {
        if ((groups + waves - 1) / waves > kWindowTileGroups) continue;
        const double us = tile_us(sh, (double)tiles, groups, waves);
        if (us < best_us) {
            best_us = us;
            best = waves;
        }
    }
    return best;
}

}  // namespace coopt
