// Windowed prefill of few rows or short streams (window.hpp), in one launch without a workspace.
//
// prefill.hip's workgroups carry 256 rows through LDS, which pays where streams are long; one that streams a stage
// or two is mostly its own start and end, a launch of few of them leaves CUs idle or needs parts and a merge, and a
// sequence of one row takes as long as one of fifty.  Here a workgroup of WAVES wavefronts takes ONE tile: 16 neighbouring
// places of a pair's list of rows by head -- three rows of five heads, or all heads of a lone row, as in decode -- so
// that its view is hardly longer than a window.  The wavefronts take the view's groups in turn, straight from the
// cache, with all but the first loads in flight under the arithmetic of attn_tile.hpp, and meet in LDS.  What bounds
// it: the tile's round trips (rows and length, block numbers, tiles) where there are few, and the L2 where there
// are many, since every tile reads its view for itself.  77 rows of 40 heads over 8 (E4M3) through 1024 + 4 tokens, 200
// tiles: 11.4 us; prefill.hip's launch 21.8, a wavefront a tile 51.
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
    int32_t num_seqs, even_tiles;       // even_tiles > 0: every sequence has so many tiles a head
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
    // Ids go round-robin over 8 XCDs.  Where 8 divides the heads, an XCD has its share of them, and a sequence's tiles of
    // a head meet in its L2; where it divides the pairs of equal sequences, an XCD has its share of these; otherwise
    // tiles are spread evenly.  (One pair of 1008 tiles on one XCD: 22 us, so 7.)
    const int id = (int)blockIdx.x, r = id >> 3;
    int g, slot, seq = 0, tile = -1;
    if ((a.H_k & 7) == 0) {
        const int share = a.H_k >> 3;
        slot = r / share;
        g = 8 * (r - slot * share) + (id & 7);
    } else if (a.even_tiles > 0 && ((a.num_seqs * a.H_k) & 7) == 0) {
        const int k = r / a.even_tiles, pair = 8 * k + (id & 7);
        seq = pair / a.H_k;
        g = pair - seq * a.H_k;
        slot = seq * a.even_tiles + r - k * a.even_tiles;
    } else {
        slot = id / a.H_k;
        g = id - slot * a.H_k;
    }
    // Slot -> sequence and tile.  A sequence that begins at row r has the slots from r G / 16 + its number on, which are
    // as many as its tiles or one more: found by 64 lanes that look at 64 of them, of the whole, then of a 64th of it.
    if (a.even_tiles > 0) {
        seq = slot / a.even_tiles;
        tile = slot - seq * a.even_tiles;
    } else {
        int left = a.num_seqs, first_slot = 0;
        while (left > 1) {
            const int step = (left + 63) >> 6, s = seq + lane * step;
            const bool in = lane * step < left;
            const int begin = in ? (int)(((long long)a.query_start[s] * a.G) >> 4) + s : 0;
            const unsigned long long before = __builtin_amdgcn_ballot_w64(in && begin <= slot);
            const int last = 63 - __builtin_clzll(before | 1ull);
            seq += last * step;
            first_slot = __builtin_amdgcn_readlane(begin, last);
            left = min(step, left - last * step);
        }
        tile = slot - first_slot;
    }
    const int qs = a.query_start[seq], C = a.query_start[seq + 1] - qs, t_ctx = a.context_lens[seq] - C;
    const int places = C * a.G, p0 = 16 * tile;
    if (tile < 0 || p0 >= places) return;
    const int at_row = p0 / a.G, last_row = min(p0 + 15, places - 1) / a.G;
    const int place = min(p0 + n, places - 1), row = place / a.G, head = g * a.G + place - row * a.G;
    half8_t q[HEAD_DIM / 32];
    load_q_operand<HEAD_DIM, KV>(q, a.q + ((size_t)(qs + row) * a.H_q + head) * HEAD_DIM, true, grp);
    // tokens up to the last row's, from the first row's window on
    const WindowView v(a.window, t_ctx + last_row + 1, t_ctx + at_row + 1 - a.window.size);
    const int nb = (v.t + kBlock - 1) / kBlock, ng = (nb + 1) >> 1;
    const int limit = t_ctx + row + 1 - v.skip * kBlock;             // the lane's column sees tokens below this
    const int seen_by_all = t_ctx + at_row + 1 - v.skip * kBlock;    // every column does
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
    const bool there = p0 + n < places;
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
        // ---- the wavefronts' sums meet: lane (n, grp) has dims 16c + 4 grp .. of place n
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
            const int c = c0 + wave;                                // dims 16c .. +15 of every place
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
                        const int32_t* block_tables, const int32_t* context_lens, const int32_t* query_start, int num_query_rows,
                        int max_chunk_len, const Window& window, void* out, const coopt_shape* sh, int waves, hipStream_t stream)
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
    a.num_seqs = sh->num_seqs;
    a.max_blocks = sh->max_blocks_per_seq;
    a.pool_tiles = sh->num_blocks * sh->num_kv_heads;
    a.window = window;
    a.scale_log2e = sh->softmax_scale * kLog2e;
    const long long slots = window_tiles(sh, num_query_rows, max_chunk_len) / sh->num_kv_heads;
    // (one sequence, or as many rows as all of them could have: no search)
    if (sh->num_seqs == 1 || (long long)num_query_rows >= (long long)sh->num_seqs * max_chunk_len)
        a.even_tiles = (int)(slots / sh->num_seqs);
    const unsigned wgs = (unsigned)(slots * sh->num_kv_heads);
    if (waves == 1) return launch_window_tiles<1>(a, sh, wgs, stream);
    if (waves == 2) return launch_window_tiles<2>(a, sh, wgs, stream);
    return launch_window_tiles<4>(a, sh, wgs, stream);
}

}  // namespace coopt
