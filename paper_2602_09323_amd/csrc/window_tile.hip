// Windowed prefill of few rows or short streams (window.hpp), in one launch without a workspace.
//
// prefill.hip's workgroups carry 256 rows through LDS, which pays where streams are long; one that streams a stage
// or two is mostly its own start and end, a launch of few of them leaves CUs idle or needs parts and a merge, and a
// sequence of one row takes as long as one of fifty.  Here a workgroup of WAVES wavefronts takes ONE tile: 16 (or 32)
// neighbouring places of a pair's list of rows by head -- three rows of five heads, or all heads of a lone row, as in decode -- so
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

// group_update (attn_tile.hpp) of SETS sets of 16 columns against one group, whose K and V are converted once for all.
template <int HEAD_DIM, int KV, int SETS>
__device__ __forceinline__ void group_update_sets(BlockRegs<HEAD_DIM, KV>& A, BlockRegs<HEAD_DIM, KV>& B,
                                                  const half8_t (&q)[SETS][HEAD_DIM / 32], float (&m)[SETS], float (&l)[SETS],
                                                  floatx4 (&acc)[SETS][HEAD_DIM / 16], bool tail, const int (&vis)[SETS], int cache,
                                                  float scale_log2e, bool any_hidden, int lo, const int (&hi)[SETS], int hi_all)
{
    float z[SETS][8];
    floatx4 sA[SETS], sB[SETS];
#pragma unroll
    for (int u = 0; u < SETS; ++u) sA[u] = sB[u] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int jj = 0; jj < HEAD_DIM / 32; ++jj) {
        const half8_t kA = k_operand<HEAD_DIM, KV>(A, jj), kB = k_operand<HEAD_DIM, KV>(B, jj);
#pragma unroll
        for (int u = 0; u < SETS; ++u) {
            sA[u] = mfma_16x16x32(kA, q[u][jj], sA[u]);
            sB[u] = mfma_16x16x32(kB, q[u][jj], sB[u]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float xA = kIsFp8<KV> ? A.ks[i] * scale_log2e : scale_log2e, xB = kIsFp8<KV> ? B.ks[i] * scale_log2e : scale_log2e;
#pragma unroll
        for (int u = 0; u < SETS; ++u) {
            z[u][i] = sA[u][i] * xA;
            z[u][4 + i] = sB[u][i] * xB;
        }
    }
    if (tail) {
        hide_tokens<HEAD_DIM, KV>(A, cache, 4);
        hide_tokens<HEAD_DIM, KV>(B, cache - kBlock, 4);
#pragma unroll
        for (int u = 0; u < SETS; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[u][i] = fminf(z[u][i], i < vis[u] ? INFINITY : -INFINITY);
                z[u][4 + i] = fminf(z[u][4 + i], i + kBlock < vis[u] ? INFINITY : -INFINITY);
            }
    }
    if (any_hidden) {
        hide_tokens<HEAD_DIM, KV>(A, lo, hi_all);
        hide_tokens<HEAD_DIM, KV>(B, lo - kBlock, hi_all - kBlock);
#pragma unroll
        for (int u = 0; u < SETS; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[u][i] = fminf(z[u][i], i >= lo && i < hi[u] ? -INFINITY : INFINITY);
                z[u][4 + i] = fminf(z[u][4 + i], i + kBlock >= lo && i + kBlock < hi[u] ? -INFINITY : INFINITY);
            }
    }
    half8_t whi[SETS], wlo[SETS];
#pragma unroll
    for (int u = 0; u < SETS; ++u) {
        const float bm = fmaxf(fmaxf(fmaxf(z[u][0], z[u][1]), fmaxf(z[u][2], z[u][3])),
                               fmaxf(fmaxf(z[u][4], z[u][5]), fmaxf(z[u][6], z[u][7])));
        if (__builtin_amdgcn_ballot_w64(bm > m[u] + kRescaleSlack) != 0) {
            float nm = fmaxf(bm, __shfl_xor(bm, 16));
            nm = fmaxf(nm, __shfl_xor(nm, 32));
            nm = fmaxf(nm, m[u]);
            const float alpha = __builtin_amdgcn_exp2f(m[u] - nm);
            l[u] *= alpha;
#pragma unroll
            for (int c = 0; c < HEAD_DIM / 16; ++c) acc[u][c] *= alpha;
            m[u] = nm;
        }
        const float mm = m[u] - kPShiftOf<KV>;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = __builtin_amdgcn_exp2f(z[u][i] - mm);
            l[u] += p[i];
        }
        if constexpr (kIsFp8<KV>) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] *= A.vs[i];
                p[4 + i] *= B.vs[i];
            }
        }
        split_weights(p, whi[u], wlo[u]);
    }
#pragma unroll
    for (int c = 0; c < HEAD_DIM / 16; ++c) {
        const half4_t va = v_operand<HEAD_DIM, KV>(A, c), vb = v_operand<HEAD_DIM, KV>(B, c);
        const half8_t v = {va[0], va[1], va[2], va[3], vb[0], vb[1], vb[2], vb[3]};
#pragma unroll
        for (int u = 0; u < SETS; ++u) {
            acc[u][c] = mfma_16x16x32(v, whi[u], acc[u][c]);
            acc[u][c] = mfma_16x16x32(v, wlo[u], acc[u][c]);
        }
    }
}

// SETS: of 16 places that a tile has.  Two share what every group costs once, its loads and the conversion of K and V, which
// pays where there are many tiles of few groups (8 x 2000 rows of 32 heads of 64 dims over 8, E4M3, through 16 tokens: 70 us,
// so 48); two groups in flight instead of three leave 64 dims three wavefronts a SIMD (of those 57, so 48).
template <int HEAD_DIM, int KV, bool BIG, int WAVES, int SETS>
__global__ void __launch_bounds__(64 * WAVES, 2)
window_tile_kernel(const WindowTileArgs a)
{
    constexpr int ES = BlockRegs<HEAD_DIM, KV>::ES;
    constexpr int DEPTH = HEAD_DIM * ES > 128 || SETS > 1 ? 2 : 3;      // groups in flight: 256 registers
    constexpr int PLACES = 16 * SETS;
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
            const int begin = in ? (int)((long long)a.query_start[s] * a.G / PLACES) + s : 0;
            const unsigned long long before = __builtin_amdgcn_ballot_w64(in && begin <= slot);
            const int last = 63 - __builtin_clzll(before | 1ull);
            seq += last * step;
            first_slot = __builtin_amdgcn_readlane(begin, last);
            left = min(step, left - last * step);
        }
        tile = slot - first_slot;
    }
    const int qs = a.query_start[seq], C = a.query_start[seq + 1] - qs, t_ctx = a.context_lens[seq] - C;
    const int places = C * a.G, p0 = PLACES * tile;
    if (tile < 0 || p0 >= places) return;
    const int at_row = p0 / a.G, last_row = min(p0 + PLACES - 1, places - 1) / a.G;
    int row[SETS];
    half_t* out[SETS];
    half8_t q[SETS][HEAD_DIM / 32];
#pragma unroll
    for (int u = 0; u < SETS; ++u) {
        const int place = min(p0 + 16 * u + n, places - 1);
        row[u] = place / a.G;
        const size_t at = ((size_t)(qs + row[u]) * a.H_q + g * a.G + place - row[u] * a.G) * HEAD_DIM;
        load_q_operand<HEAD_DIM, KV>(q[u], a.q + at, true, grp);
        out[u] = a.out + at + 4 * grp;
    }
    // tokens up to the last row's, from the first row's window on
    const WindowView v(a.window, t_ctx + last_row + 1, t_ctx + at_row + 1 - a.window.size);
    const int nb = (v.t + kBlock - 1) / kBlock, ng = (nb + 1) >> 1;
    int limit[SETS];                                                 // the lane's columns see tokens below this
#pragma unroll
    for (int u = 0; u < SETS; ++u) limit[u] = t_ctx + row[u] + 1 - v.skip * kBlock;
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
    float m[SETS], l[SETS];
    floatx4 acc[SETS][HEAD_DIM / 16];
#pragma unroll
    for (int u = 0; u < SETS; ++u) {
        m[u] = kNoScore;
        l[u] = 0.0f;
#pragma unroll
        for (int c = 0; c < HEAD_DIM / 16; ++c) acc[u][c] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
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
                const bool any_hidden = base < v.hi + PLACES - 1 && base + 2 * kBlock > v.lo, tail = base + 2 * kBlock > seen_by_all;
                if constexpr (SETS == 1) {
                    const Hole hole{any_hidden, v.lo - at, limit[0] - a.window.size - at, v.hi - at};
                    group_update<HEAD_DIM, KV, true>(regs[u][0], regs[u][1], q[0], m[0], l[0], acc[0], tail, limit[0] - at,
                                                     limit[0] - at - kBlock, v.t - at, v.t - at - kBlock, a.scale_log2e, hole);
                } else {
                    int vis[SETS], hi[SETS];
#pragma unroll
                    for (int w = 0; w < SETS; ++w) {
                        vis[w] = limit[w] - at;
                        hi[w] = limit[w] - a.window.size - at;
                    }
                    group_update_sets<HEAD_DIM, KV, SETS>(regs[u][0], regs[u][1], q, m, l, acc, tail, vis, v.t - at, a.scale_log2e,
                                                          any_hidden, v.lo - at, hi, v.hi - at);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            issue(regs[u], e + DEPTH);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int u = 0; u < SETS; ++u) {
        l[u] += __shfl_xor(l[u], 16);
        l[u] += __shfl_xor(l[u], 32);
    }
    // (the caller's rows may begin at any 2-byte boundary)
    typedef _Float16 row_piece_t __attribute__((ext_vector_type(4), aligned(2)));
    auto store = [&](int u, int c, floatx4 o, float inv) {
        if (p0 + 16 * u + n < places)
            *reinterpret_cast<row_piece_t*>(out[u] + 16 * c) =
                row_piece_t{(half_t)(o[0] * inv), (half_t)(o[1] * inv), (half_t)(o[2] * inv), (half_t)(o[3] * inv)};
    };
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int u = 0; u < SETS; ++u) {
            const float inv = 1.0f / l[u];
#pragma unroll
            for (int c = 0; c < HEAD_DIM / 16; ++c) store(u, c, acc[u][c], inv);
        }
    } else {
        static_assert(SETS == 1);
        // ---- the wavefronts' sums meet: lane (n, grp) has dims 16c + 4 grp .. of place n
        __shared__ __attribute__((aligned(16))) unsigned char sums[WAVES][HEAD_DIM / 16 * 1024 + 512];
        constexpr int kML = HEAD_DIM / 16 * 1024;
#pragma unroll
        for (int c = 0; c < HEAD_DIM / 16; ++c) *reinterpret_cast<floatx4*>(sums[wave] + 1024 * c + 16 * lane) = acc[0][c];
        *reinterpret_cast<float*>(sums[wave] + kML + 4 * lane) = m[0];
        *reinterpret_cast<float*>(sums[wave] + kML + 256 + 4 * lane) = l[0];
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
            store(0, c, o, inv);
        }
    }
}

template <int WAVES, int SETS>
static int launch_window_tiles(const WindowTileArgs& a, const coopt_shape* sh, unsigned wgs, hipStream_t stream)
{
    const bool big = !pool_fits_small(sh);
    auto launch = [&](auto dim, auto kv) {
        constexpr int D = decltype(dim)::value, KV = decltype(kv)::value;
        if (big) hipLaunchKernelGGL((window_tile_kernel<D, KV, true, WAVES, SETS>), dim3(wgs), dim3(64 * WAVES), 0, stream, a);
        else hipLaunchKernelGGL((window_tile_kernel<D, KV, false, WAVES, SETS>), dim3(wgs), dim3(64 * WAVES), 0, stream, a);
    };
    auto of_dim = [&](auto kv) {
        if (sh->head_dim == 128) {
            if constexpr (SETS == 1 || decltype(kv)::value != COOPT_KV_FP16) launch(std::integral_constant<int, 128>{}, kv);
        } else launch(std::integral_constant<int, 64>{}, kv);
    };
    if (sh->kv_dtype == COOPT_KV_E4M3) of_dim(std::integral_constant<int, COOPT_KV_E4M3>{});
    else if (sh->kv_dtype == COOPT_KV_E5M2) of_dim(std::integral_constant<int, COOPT_KV_E5M2>{});
    else of_dim(std::integral_constant<int, COOPT_KV_FP16>{});
    return launch_status();
}

int launch_window_tiles(const void* q, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                        const int32_t* block_tables, const int32_t* context_lens, const int32_t* query_start, int num_query_rows,
                        int max_chunk_len, const Window& window, void* out, const coopt_shape* sh, int waves, int sets, hipStream_t stream)
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
    const long long slots = window_tiles(sh, num_query_rows, max_chunk_len, 16 * sets) / sh->num_kv_heads;
    // (one sequence, or as many rows as all of them could have: no search)
    if (sh->num_seqs == 1 || (long long)num_query_rows >= (long long)sh->num_seqs * max_chunk_len)
        a.even_tiles = (int)(slots / sh->num_seqs);
    const unsigned wgs = (unsigned)(slots * sh->num_kv_heads);
    if (sets == 2) return launch_window_tiles<1, 2>(a, sh, wgs, stream);
    if (waves == 1) return launch_window_tiles<1, 1>(a, sh, wgs, stream);
    if (waves == 2) return launch_window_tiles<2, 1>(a, sh, wgs, stream);
    return launch_window_tiles<4, 1>(a, sh, wgs, stream);
}

}  // namespace coopt
