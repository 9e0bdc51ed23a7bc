// Windowed prefill of few or short streams (window.hpp), in one launch without a workspace.
//
// prefill.hip's workgroups carry 256 rows through LDS, which pays where streams are long; one that streams a stage
// or two is mostly its own start and end, and a launch of few of them leaves CUs idle or needs parts and a merge.
// Here a workgroup of WAVES wavefronts takes ONE tile, 16 rows of a head: the wavefronts take the groups of the tile's
// view in turn, straight from the cache, with all but the first loads in flight under the arithmetic of
// attn_tile.hpp, and meet in LDS.  What bounds it: the tile's round trips (rows and length, block numbers, tiles)
// where there are few, and the L2 where there are many, since every tile reads its view for itself: a pair's
// tiles sit on one XCD.
#include "attn_tile.hpp"
#include "window_tile.hpp"

namespace coopt {

struct WindowTileArgs {
    const half_t* q;
    CacheView cv;
    const int32_t* block_tables;
    const int32_t* context_lens;
    const int32_t* query_start;
    half_t* out;
    int32_t H_q, H_k, G;
    int32_t num_pairs, pair_tiles;      // tiles of a pair: rows, then heads
    int32_t max_blocks, pool_tiles;
    Window window;
    float scale_log2e;
};

template <int HEAD_DIM, int KV, bool BIG, int WAVES>
__global__ void __launch_bounds__(64 * WAVES, 2)
window_tile_kernel(const WindowTileArgs a)
{
    constexpr int ES = BlockRegs<HEAD_DIM, KV>::ES;
    constexpr int DEPTH = HEAD_DIM * ES > 128 ? 2 : 3;      // groups in flight: 256 registers
    const int lane = threadIdx.x & 63, wave = wave_uniform((int)(threadIdx.x >> 6)), n = lane & 15, grp = lane >> 4;
    // Ids go round-robin over 8 XCDs.  Where 8 divides the pairs, an XCD takes its share of them one after the other, all
    // of a pair's tiles; otherwise tile by tile, which spreads the pairs evenly.  (One pair of 1008 tiles on
    // one XCD: 22 us, so 7.)
    const int id = (int)blockIdx.x;
    int pair, tile;
    if ((a.num_pairs & 7) == 0) {
        const int k = (id >> 3) / a.pair_tiles;
        tile = (id >> 3) - k * a.pair_tiles;
        pair = 8 * k + (id & 7);
    } else {
        tile = id / a.num_pairs;
        pair = id - tile * a.num_pairs;
    }
    const int seq = pair / a.H_k, g = pair - seq * a.H_k;
    const int i0 = 16 * (tile / a.G), head = g * a.G + tile % a.G;
    const int qs = a.query_start[seq], C = a.query_start[seq + 1] - qs, t_ctx = a.context_lens[seq] - C;
    if (i0 >= C) return;
    const int row = min(i0 + n, C - 1);
    half8_t q[HEAD_DIM / 32];
    load_q_operand<HEAD_DIM, KV>(q, a.q + ((size_t)(qs + row) * a.H_q + head) * HEAD_DIM, true, grp);
    // tokens up to the last row's, from the first row's window on
    const WindowView v(a.window, t_ctx + min(i0 + 15, C - 1) + 1, t_ctx + i0 + 1 - a.window.size);
    const int nb = (v.t + kBlock - 1) / kBlock, ng = (nb + 1) >> 1;
    const int limit = t_ctx + row + 1 - v.skip * kBlock;             // the lane's column sees tokens below this
    const int seen_by_all = t_ctx + i0 + 1 - v.skip * kBlock;        // every column does
    const int* bt = a.block_tables + (size_t)seq * a.max_blocks;
    auto group_of = [&](int e) { return e * WAVES + wave; };
    const int count = wave < ng ? min((ng - wave - 1) / WAVES + 1, kWindowTileGroups) : 0;
    // lane 2e + h: block h of the wavefront's group e, and of its group 32 + e
    auto id_at = [&](int e) {
        const int b = 2 * group_of(e) + (lane & 1);
        return b < nb && v.block(b) < a.max_blocks ? bt[v.block(b)] : 0;
    };
    const int ids = id_at(lane >> 1), ids_on = id_at(32 + (lane >> 1));

    const TileLoader<HEAD_DIM, KV, BIG> loader(a.cv, lane, a.pool_tiles);
    BlockRegs<HEAD_DIM, KV> regs[DEPTH][2];
    auto issue = [&](BlockRegs<HEAD_DIM, KV> (&r)[2], int e) {
        const int b = 2 * group_of(e), at = 2 * (e & 31);
        const int idA = e < 32 ? __builtin_amdgcn_readlane(ids, at) : __builtin_amdgcn_readlane(ids_on, at);
        const int idB = e < 32 ? __builtin_amdgcn_readlane(ids, at + 1) : __builtin_amdgcn_readlane(ids_on, at + 1);
        loader.issue(r[0], e < count ? idA * a.H_k + g : g, e < count);
        loader.issue(r[1], e < count && b + 1 < nb ? idB * a.H_k + g : g, e < count && b + 1 < nb);
    };
    // (finite: a column may see nothing of a wavefront's groups)
    float m = -0x1.fffffep127f, l = 0.0f;
    floatx4 acc[HEAD_DIM / 16];
#pragma unroll
    for (int c = 0; c < HEAD_DIM / 16; ++c) acc[c] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) {
        issue(regs[u], u);
        __builtin_amdgcn_sched_barrier(0);
    }
    for (int j = 0; j < count; j += DEPTH) {
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            const int e = j + u;
            if (e < count) {
                const int base = 2 * kBlock * group_of(e), at = base + 4 * grp;
                const Hole hole{base < v.hi + 15 && base + 2 * kBlock > v.lo, v.lo - at, limit - a.window.size - at, v.hi - at};
                group_update<HEAD_DIM, KV, true>(regs[u][0], regs[u][1], q, m, l, acc, base + 2 * kBlock > seen_by_all, limit - at,
                                                 limit - at - kBlock, v.t - at, v.t - at - kBlock, a.scale_log2e, hole);
            }
            __builtin_amdgcn_sched_barrier(0);
            issue(regs[u], e + DEPTH);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    half_t* out = a.out + ((size_t)(qs + row) * a.H_q + head) * HEAD_DIM + 4 * grp;
    const bool there = i0 + n < C;
    // (the caller's rows may begin at any 2-byte boundary)
    typedef _Float16 row_piece_t __attribute__((ext_vector_type(4), aligned(2)));
    auto store = [&](int c, floatx4 o, float inv) {
        if (there)
            *reinterpret_cast<row_piece_t*>(out + 16 * c) =
                row_piece_t{(half_t)(o[0] * inv), (half_t)(o[1] * inv), (half_t)(o[2] * inv), (half_t)(o[3] * inv)};
    };
    if constexpr (WAVES == 1) {
        const float inv = 1.0f / l;
#pragma unroll
        for (int c = 0; c < HEAD_DIM / 16; ++c) store(c, acc[c], inv);
    } else {
        // ---- the wavefronts' sums meet: lane (n, grp) has dims 16c + 4 grp .. of row n
        __shared__ __attribute__((aligned(16))) unsigned char sums[WAVES][HEAD_DIM / 16 * 1024 + 512];
        constexpr int kML = HEAD_DIM / 16 * 1024;
#pragma unroll
        for (int c = 0; c < HEAD_DIM / 16; ++c) *reinterpret_cast<floatx4*>(sums[wave] + 1024 * c + 16 * lane) = acc[c];
        *reinterpret_cast<float*>(sums[wave] + kML + 4 * lane) = m;
        *reinterpret_cast<float*>(sums[wave] + kML + 256 + 4 * lane) = l;
        __syncthreads();
        float x[WAVES], M = -INFINITY, L = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            x[w] = *reinterpret_cast<const float*>(sums[w] + kML + 4 * lane);
            M = fmaxf(M, x[w]);
        }
        // (a wavefront without groups is left out, not weighted by zero)
        const int had = min(ng, WAVES);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            x[w] = __builtin_amdgcn_exp2f(x[w] - M);
            L += w < had ? *reinterpret_cast<const float*>(sums[w] + kML + 256 + 4 * lane) * x[w] : 0.0f;
        }
        const float inv = 1.0f / L;
#pragma unroll
        for (int c0 = 0; c0 < HEAD_DIM / 16; c0 += WAVES) {
            const int c = c0 + wave;                                // dims 16c .. +15 of every row
            if (c >= HEAD_DIM / 16) break;
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const floatx4 s = *reinterpret_cast<const floatx4*>(sums[w] + 1024 * c + 16 * lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += w < had ? s[i] * x[w] : 0.0f;
            }
            store(c, o, inv);
        }
    }
}

template <int WAVES>
static int launch_window_tiles(const WindowTileArgs& a, const coopt_shape* sh, unsigned wgs, hipStream_t stream)
{
    const bool big = !pool_fits_small(sh);
    auto launch = [&](auto dim, auto kv) {
        constexpr int D = decltype(dim)::value, KV = decltype(kv)::value;
        if (big) hipLaunchKernelGGL((window_tile_kernel<D, KV, true, WAVES>), dim3(wgs), dim3(64 * WAVES), 0, stream, a);
        else hipLaunchKernelGGL((window_tile_kernel<D, KV, false, WAVES>), dim3(wgs), dim3(64 * WAVES), 0, stream, a);
    };
    auto of_dim = [&](auto kv) {
        if (sh->head_dim == 128) launch(std::integral_constant<int, 128>{}, kv);
        else launch(std::integral_constant<int, 64>{}, kv);
    };
    if (sh->kv_dtype == COOPT_KV_E4M3) of_dim(std::integral_constant<int, COOPT_KV_E4M3>{});
    else if (sh->kv_dtype == COOPT_KV_E5M2) of_dim(std::integral_constant<int, COOPT_KV_E5M2>{});
    else of_dim(std::integral_constant<int, COOPT_KV_FP16>{});
    return launch_status();
}

int launch_window_tiles(const void* q, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                        const int32_t* block_tables, const int32_t* context_lens, const int32_t* query_start, int max_chunk_len,
                        const Window& window, void* out, const coopt_shape* sh, int waves, hipStream_t stream)
{
    WindowTileArgs a{};
    a.q = (const half_t*)q;
    a.cv = CacheView{(const uint8_t*)k_cache, (const uint8_t*)v_cache, k_scale, v_scale};
    a.block_tables = block_tables;
    a.context_lens = context_lens;
    a.query_start = query_start;
    a.out = (half_t*)out;
    a.H_q = sh->num_q_heads;
    a.H_k = sh->num_kv_heads;
    a.G = sh->num_q_heads / sh->num_kv_heads;
    a.num_pairs = sh->num_seqs * sh->num_kv_heads;
    a.max_blocks = sh->max_blocks_per_seq;
    a.pool_tiles = sh->num_blocks * sh->num_kv_heads;
    a.window = window;
    a.scale_log2e = sh->softmax_scale * kLog2e;
    a.pair_tiles = a.G * ((max_chunk_len + 15) / 16);
    const unsigned wgs = (unsigned)a.num_pairs * (unsigned)a.pair_tiles;
    if (waves == 1) return launch_window_tiles<1>(a, sh, wgs, stream);
    if (waves == 2) return launch_window_tiles<2>(a, sh, wgs, stream);
    return launch_window_tiles<4>(a, sh, wgs, stream);
}

}  // namespace coopt
