// Attention through a sliding window with the sequence's first tokens visible (window.hpp), over the paged
// cache.  Per query row it is Background Eq. 1 over the tokens that the row sees, with the grouping of
// Opt-GQA Eq. 7 and the running softmax of Opt-Pa Eq. 10; the per-group arithmetic is in attn_tile.hpp.
//
// One wavefront takes one column tile -- decode: the query heads of a (sequence, KV head) pair; prefill: 16
// rows of a head -- and streams its view of the sequence, two blocks at a time.
#include "attn_tile.hpp"
#include "launch_grid.hpp"
#include "window.hpp"

namespace coopt {

struct WindowArgs {
    const half_t* q;
    CacheView cv;
    const int32_t* block_tables;
    const int32_t* context_lens;
    const int32_t* query_start;      // prefill only
    half_t* out;
    int32_t H_q, H_k, G;
    int32_t max_blocks, pool_tiles;
    int32_t tiles;                   // prefill: tiles of 16 rows per head
    Window window;
    float scale_log2e;
};

// limit, lower: what the lane's column sees of the view, tokens below `limit` and not in [lo, lower); no column
// has a lower above `hidden`.
template <int HEAD_DIM, int KV, bool BIG>
__device__ __forceinline__ void stream_view(const WindowArgs& a, const WindowView& v, int seq, int g, int limit, int lower, int hidden,
                                            const half8_t (&q)[HEAD_DIM / 32], floatx4 (&acc)[HEAD_DIM / 16], float& l, int lane)
{
    const int grp = lane >> 4;
    const TileLoader<HEAD_DIM, KV, BIG> loader(a.cv, lane, a.pool_tiles);
    const int32_t* bt = a.block_tables + (size_t)seq * a.max_blocks;
    const int nb = (v.t + kBlock - 1) / kBlock;
    // (finite: a column may see nothing of the first groups)
    float m = -0x1.fffffep127f;
#pragma unroll
    for (int c = 0; c < HEAD_DIM / 16; ++c) acc[c] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int b = 0; b < nb; b += 2) {
        BlockRegs<HEAD_DIM, KV> A, B;
        const bool two = b + 1 < nb;
        loader.issue(A, wave_uniform(bt[v.block(b)]) * a.H_k + g, true);
        loader.issue(B, two ? wave_uniform(bt[v.block(b + 1)]) * a.H_k + g : 0, two);
        const int base = kBlock * b + 4 * grp;
        const Hole hole{kBlock * b < hidden, v.lo - base, lower - base, v.hi - base};
        group_update<HEAD_DIM, KV, true>(A, B, q, m, l, acc, true, limit - base, limit - base - kBlock, v.t - base,
                                         v.t - base - kBlock, a.scale_log2e, hole);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
}

template <int HEAD_DIM, int KV, bool BIG>
__global__ void __launch_bounds__(64)
window_prefill_kernel(const WindowArgs a)
{
    const int lane = threadIdx.x, n = lane & 15, grp = lane >> 4;
    const int tile = blockIdx.x % a.tiles, at = blockIdx.x / a.tiles, seq = at / a.H_q, head = at - seq * a.H_q;
    const int qs = a.query_start[seq], C = a.query_start[seq + 1] - qs, t_ctx = a.context_lens[seq] - C;
    if (16 * tile >= C) return;
    const int row = min(16 * tile + n, C - 1), last = min(16 * tile + 15, C - 1);
    half8_t q[HEAD_DIM / 32];
    load_q_operand<HEAD_DIM, KV>(q, a.q + ((size_t)(qs + row) * a.H_q + head) * HEAD_DIM, true, grp);
    // tokens up to the tile's last row's, from the window of its first row on
    const WindowView v(a.window, t_ctx + last + 1, t_ctx + 16 * tile + 1 - a.window.size);
    const int limit = t_ctx + row + 1 - v.skip * kBlock;
    floatx4 acc[HEAD_DIM / 16];
    float l = 0.0f;
    stream_view<HEAD_DIM, KV, BIG>(a, v, seq, head / a.G, limit, limit - a.window.size, v.hi + 15, q, acc, l, lane);
    if (16 * tile + n >= C) return;
    const float inv = 1.0f / l;
    half_t* out = a.out + ((size_t)(qs + row) * a.H_q + head) * HEAD_DIM + 4 * grp;
#pragma unroll
    for (int c = 0; c < HEAD_DIM / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) out[16 * c + i] = (half_t)(acc[c][i] * inv);
}

}  // namespace coopt

using namespace coopt;

static WindowArgs window_args(const void* q, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                              const int32_t* block_tables, const int32_t* context_lens, int window, int num_sinks, void* out,
                              const coopt_shape* sh)
{
    WindowArgs a{};
    a.q = (const half_t*)q;
    a.cv = CacheView{(const uint8_t*)k_cache, (const uint8_t*)v_cache, k_scale, v_scale};
    a.block_tables = block_tables;
    a.context_lens = context_lens;
    a.out = (half_t*)out;
    a.H_q = sh->num_q_heads;
    a.H_k = sh->num_kv_heads;
    a.G = sh->num_q_heads / sh->num_kv_heads;
    a.max_blocks = sh->max_blocks_per_seq;
    a.pool_tiles = sh->num_blocks * sh->num_kv_heads;
    a.window = window_of(sh, window, num_sinks);
    a.scale_log2e = sh->softmax_scale * kLog2e;
    return a;
}

template <class F>
static void for_cache(const coopt_shape* sh, F launch)
{
    const bool big = !pool_fits_small(sh);
    auto of_dim = [&](auto kv) {
        if (sh->head_dim == 128) big ? launch(std::integral_constant<int, 128>{}, kv, std::true_type{}) : launch(std::integral_constant<int, 128>{}, kv, std::false_type{});
        else big ? launch(std::integral_constant<int, 64>{}, kv, std::true_type{}) : launch(std::integral_constant<int, 64>{}, kv, std::false_type{});
    };
    if (sh->kv_dtype == COOPT_KV_E4M3) of_dim(std::integral_constant<int, COOPT_KV_E4M3>{});
    else if (sh->kv_dtype == COOPT_KV_E5M2) of_dim(std::integral_constant<int, COOPT_KV_E5M2>{});
    else of_dim(std::integral_constant<int, COOPT_KV_FP16>{});
}

extern "C" size_t coopt_prefill_window_workspace_bytes(const coopt_shape* sh, int32_t max_chunk_len, int32_t window, int32_t num_sinks)
{
    return 0;
}

extern "C" int coopt_paged_gqa_prefill_chunk_window(const void* q, const void* k_cache, const void* v_cache, const float* k_scale,
                                                    const float* v_scale, const int32_t* block_tables,
                                                    const int32_t* context_lens, const int32_t* query_start,
                                                    int32_t num_query_rows, int32_t max_chunk_len, int32_t window,
                                                    int32_t num_sinks, void* out, void* workspace, size_t workspace_bytes,
                                                    const coopt_shape* sh, void* hip_stream)
{
    int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    st = check_window(window, num_sinks);
    if (st != COOPT_OK) return st;
    if (num_query_rows < 0 || max_chunk_len < 0) return COOPT_ERR_SHAPE;
    if (sh->num_seqs == 0 || num_query_rows == 0 || max_chunk_len == 0) return COOPT_OK;
    if (!q || !k_cache || !v_cache || !block_tables || !context_lens || !query_start || !out) return COOPT_ERR_NULL;
    if (sh->kv_dtype != COOPT_KV_FP16 && (!k_scale || !v_scale)) return COOPT_ERR_NULL;
    WindowArgs a = window_args(q, k_cache, v_cache, k_scale, v_scale, block_tables, context_lens, window, num_sinks, out, sh);
    a.query_start = query_start;
    a.tiles = (max_chunk_len + 15) / 16;
    const long long wgs = (long long)sh->num_seqs * sh->num_q_heads * a.tiles;
    if (wgs > 4 * kMaxWorkgroups) return COOPT_ERR_SHAPE;
    for_cache(sh, [&](auto dim, auto kv, auto big) {
        hipLaunchKernelGGL((window_prefill_kernel<decltype(dim)::value, decltype(kv)::value, decltype(big)::value>),
                           dim3((unsigned)wgs), dim3(64), 0, (hipStream_t)hip_stream, a);
    });
    return launch_status();
}
