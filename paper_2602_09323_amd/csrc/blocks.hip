// The pool's blocks as whole numbers: who holds them, which are free, and moving them about.
//
// A block is free where no table entry names it; the map of free blocks holds one bit a block, so that
// the lowest free ones are found by counting bits (a pool of 200 000 blocks: 25 KB), whatever was freed before
// and in which order.  Every call takes blocks in that order, which makes its results the same every time
// although references are counted with atomics.
//
// The calls are a few KB of integers: what bounds them is launches and memory round trips, not bytes.
// What has to be agreed on by all sequences (how many blocks are needed, which are the lowest free ones) is one
// workgroup of 16 wavefronts; what is done row by row is a second launch where there are rows enough.  Copying
// is bound by HBM.  In us, of few entries / of the largest case measured: free 2.1 / 4.5 (64 sequences of up to 219 blocks),
// behind a window 2.2 / 3.4 (1024 sequences), reserve 3.8 (16) / 9.8 + 3.8 for the slots (1024, 4151 new blocks, 66 416
// rows), fork 5.9 / 5.9 + 4.5 (128 children of up to 250 blocks), compact 6 / 10.4 + 4.7 (a pool of 18 225 blocks).
#include <type_traits>

#include "common.hpp"
#include "launch_grid.hpp"

namespace coopt {

constexpr int kPlanThreads = 1024;             // of the workgroup that plans
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kListed = 8192;                  // new blocks kept in LDS; more go to the workspace
constexpr long long kFewEntries = 8192;        // table entries that the planning workgroup works on itself: a second launch
                                               // takes longer (8 forks of 44 entries: 5.7 + 3.6 us, 6.0 so)

// Where a call's parts lie in the workspace (32-bit words).
struct BlocksWorkspace {
    int32_t* list;      // [num_blocks] new blocks, lowest first; compact: the new place of every block
    int32_t* first;     // [num_seqs] place in the list of a sequence's first new block; fork: tokens of the parents
    int32_t* used;      // compact: blocks in use
};
constexpr int kBlocksHeaderWords = 16;

inline size_t blocks_workspace_bytes(const coopt_shape* sh)
{
    return 4 * ((size_t)kBlocksHeaderWords + sh->num_blocks + sh->num_seqs);
}
inline BlocksWorkspace blocks_workspace(void* at, const coopt_shape* sh)
{
    int32_t* w = (int32_t*)at;
    return BlocksWorkspace{w + kBlocksHeaderWords, w + kBlocksHeaderWords + sh->num_blocks, w};
}

struct BlocksArgs {
    int32_t* tables;
    int32_t* lens;
    int32_t* refs;
    uint32_t* free_map;
    BlocksWorkspace ws;
    int32_t num_seqs, max_blocks, num_blocks, words;
};

__device__ __forceinline__ int blocks_of(int tokens) { return (tokens + kBlock - 1) / kBlock; }
__device__ __forceinline__ bool is_block(const BlocksArgs& a, int id) { return (uint32_t)id < (uint32_t)a.num_blocks; }

// One reference less; the last one frees the block.
__device__ __forceinline__ void release(const BlocksArgs& a, int id)
{
    if (is_block(a, id) && atomicSub(a.refs + id, 1) == 1) atomicOr(a.free_map + (id >> 5), 1u << (id & 31));
}

// Exclusive prefix sum over the workgroup's threads, and the total.  (sums: one of each wavefront)
__device__ __forceinline__ int plan_scan(int v, int* sums, int& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int incl = wave_inclusive_scan(v);
    __syncthreads();                            // (the sums of the scan before this one have been read)
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    const int mine = wave_inclusive_scan(lane < kPlanWaves ? sums[lane] : 0);
    total = __builtin_amdgcn_readlane(mine, kPlanWaves - 1);
    return incl - v + (wave > 0 ? __shfl(mine, max(wave - 1, 0)) : 0);
}

// Bits of word w of the map that are blocks below x.
__device__ __forceinline__ uint32_t bits_below(int w, int x)
{
    const long long n = x - 32LL * w;
    return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
}
__device__ __forceinline__ uint32_t free_word(const BlocksArgs& a, int w)
{
    return w < a.words ? a.free_map[w] & bits_below(w, a.num_blocks) : 0u;
}

// The `need` lowest free blocks, into list[0 .. need-1], and out of the map with a reference each -- or, where
// there are fewer, nothing but how many are missing.  first_word: the thread's word of the map's first; cut: a
// word of LDS.
__device__ __forceinline__ int take_blocks(const BlocksArgs& a, uint32_t first_word, int need, int* list, int* sums, int* cut)
{
    if (need <= 0) return 0;
    int have = 0, base = 0;
    for (; base < a.words && have < need; base += kPlanThreads) {
        const int w = base + threadIdx.x;
        uint32_t bits = base == 0 ? first_word : free_word(a, w);
        int total, at = have + plan_scan(__builtin_popcount(bits), sums, total);
        if (at < need && at + __builtin_popcount(bits) >= need) *cut = w;          // the last word that is taken from
        for (; bits && at < need; ++at, bits &= bits - 1) list[at] = 32 * w + __builtin_ctz(bits);
        have += total;
    }
    __syncthreads();
    if (have < need) return need - have;
    const int last = *cut, top = list[need - 1];
    for (int w = threadIdx.x; w < last; w += kPlanThreads) a.free_map[w] = 0u;
    if (threadIdx.x == 0) a.free_map[last] &= ~(0xffffffffu >> (31 - (top & 31)));
    for (int r = threadIdx.x; r < need; r += kPlanThreads) a.refs[list[r]] = 1;
    return 0;
}

// The last of n entries of an increasing array (from its first, 0) that is not above x.
template <class At>
__device__ __forceinline__ int last_not_above(int n, int x, At at)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at(mid) <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---- the state of a pool from its tables

__global__ void __launch_bounds__(256)
blocks_clear_kernel(const BlocksArgs a)
{
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < a.num_blocks; i += gridDim.x * 256LL) a.refs[i] = 0;
}

__global__ void __launch_bounds__(256)
blocks_count_kernel(const BlocksArgs a)
{
    const int nb = min(blocks_of(max(a.lens[blockIdx.x], 0)), a.max_blocks);
    const int32_t* row = a.tables + (size_t)blockIdx.x * a.max_blocks;
    for (int b = threadIdx.x; b < nb; b += 256)
        if (is_block(a, row[b])) atomicAdd(a.refs + row[b], 1);
}

__global__ void __launch_bounds__(256)
blocks_map_kernel(const BlocksArgs a)
{
    for (long long base = (blockIdx.x * 4LL + (threadIdx.x >> 6)) * 64; base < a.num_blocks; base += gridDim.x * 256LL) {
        const int lane = threadIdx.x & 63;
        const long long id = base + lane;
        const unsigned long long bits = __builtin_amdgcn_ballot_w64(id < a.num_blocks && a.refs[id] == 0);
        if (lane < 2 && base / 32 + lane < a.words) a.free_map[base / 32 + lane] = (uint32_t)(bits >> (32 * lane));
    }
}

// ---- freeing

// A workgroup per listed sequence: its length is taken out first, so that the same index twice frees once.
__global__ void __launch_bounds__(1024)
blocks_free_kernel(const BlocksArgs a, const int32_t* seqs)
{
    __shared__ int tokens;
    const int s = seqs[blockIdx.x];
    if ((uint32_t)s >= (uint32_t)a.num_seqs) return;
    if (threadIdx.x == 0) tokens = atomicExch(a.lens + s, 0);
    __syncthreads();
    const int nb = min(blocks_of(max(tokens, 0)), a.max_blocks);
    for (int b = threadIdx.x; b < nb; b += blockDim.x) release(a, a.tables[(size_t)s * a.max_blocks + b]);
}

// A wavefront per sequence, from the window down: what earlier calls have freed (-1) lies below, so
// the walk ends at the first of it.
__global__ void __launch_bounds__(256)
blocks_free_window_kernel(const BlocksArgs a, int window, int sinks)
{
    const int s = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (s >= a.num_seqs) return;
    int32_t* row = a.tables + (size_t)s * a.max_blocks;
    const int lead = (sinks + kBlock - 1) / kBlock;
    for (int top = min((a.lens[s] - window) / kBlock, a.max_blocks); top > lead; top -= 64) {
        const int b = top - 1 - lane;
        const int id = b >= lead ? row[b] : 0;
        if (b >= lead && is_block(a, id)) {        // (another entry is not the sequence's)
            release(a, id);
            row[b] = -1;
        }
        if (__builtin_amdgcn_ballot_w64(id == -1)) break;
    }
}

// ---- room for new tokens

// Rows of sequence s: query_start's, or one of every sequence that holds tokens.
__device__ __forceinline__ int new_tokens(const BlocksArgs& a, const int32_t* starts, int s, int t)
{
    return starts ? starts[s + 1] - starts[s] : t > 0 ? 1 : 0;
}

__device__ __forceinline__ int64_t slot_of(const BlocksArgs& a, int s, int pos)
{
    return (int64_t)a.tables[(size_t)s * a.max_blocks + pos / kBlock] * kBlock + pos % kBlock;
}

// Where nothing is reserved, no row keeps a slot that a write would take: -1, also over what an earlier step left in
// the rows behind the last sequence's (which a reservation leaves alone; negative ones stay).
__device__ __forceinline__ void refuse_slot(int64_t* slots, int r, int rows)
{
    if (r < rows || slots[r] >= 0) slots[r] = -1;
}

// SLOTS: the rows' slots, too (few rows; else blocks_slots_kernel behind this).
template <bool SLOTS>
__global__ void __launch_bounds__(kPlanThreads)
blocks_reserve_kernel(const BlocksArgs a, const int32_t* starts, int num_rows, int64_t* slots, int32_t* result)
{
    __shared__ int sums[kPlanWaves], cut, refused, listed[kListed], first_listed[kPlanThreads];
    if (threadIdx.x == 0) refused = starts && (starts[0] != 0 || starts[a.num_seqs] > num_rows);
    const uint32_t word = free_word(a, threadIdx.x);        // (asked for with the lengths)
    int* first = a.num_seqs <= kPlanThreads ? first_listed : a.ws.first;
    int need = 0;
    __syncthreads();
    for (int base = 0; base < a.num_seqs; base += kPlanThreads) {
        const int s = base + threadIdx.x;
        int mine = 0;
        if (s < a.num_seqs) {
            const int t = a.lens[s], n = new_tokens(a, starts, s, t);
            if (n < 0 || t < 0 || (long long)t + n > (long long)a.max_blocks * kBlock) refused = 1;
            else mine = blocks_of(t + n) - blocks_of(t);
        }
        int total;
        const int before = plan_scan(mine, sums, total);
        if (s < a.num_seqs) first[s] = need + before;
        need += total;
    }
    __syncthreads();
    int* list = need <= kListed ? listed : a.ws.list;
    const int missing = refused ? -1 : take_blocks(a, word, need, list, sums, &cut);
    if (threadIdx.x == 0) *result = missing;
    const int rows = starts ? min(max(starts[a.num_seqs], 0), num_rows) : a.num_seqs;
    if (missing != 0) {
        if (SLOTS)
            for (int r = threadIdx.x; r < num_rows; r += kPlanThreads) refuse_slot(slots, r, rows);
        return;
    }
    // the new blocks' places in the tables
    for (int r = threadIdx.x; r < need; r += kPlanThreads) {
        const int s = last_not_above(a.num_seqs, r, [&](int i) { return first[i]; });
        a.tables[(size_t)s * a.max_blocks + blocks_of(a.lens[s]) + r - first[s]] = list[r];
    }
    __syncthreads();
    if constexpr (SLOTS) {
        for (int r = threadIdx.x; r < rows; r += kPlanThreads) {
            const int s = starts ? last_not_above(a.num_seqs, r, [&](int i) { return starts[i]; }) : r;
            const int t = a.lens[s];
            slots[r] = starts || t > 0 ? slot_of(a, s, t + (starts ? r - starts[s] : 0)) : -1;
        }
        __syncthreads();
    }
    for (int s = threadIdx.x; s < a.num_seqs; s += kPlanThreads) a.lens[s] += new_tokens(a, starts, s, a.lens[s]);
}

// The slots of many rows, from the tables and lengths as the reservation has left them.
__global__ void __launch_bounds__(256)
blocks_slots_kernel(const BlocksArgs a, const int32_t* starts, int num_rows, int64_t* slots, const int32_t* result)
{
    const int r = blockIdx.x * 256 + threadIdx.x;
    const int rows = starts ? min(starts[a.num_seqs], num_rows) : a.num_seqs;
    if (r >= num_rows) return;
    if (*result != 0) {
        refuse_slot(slots, r, rows);
        return;
    }
    if (r >= rows) return;
    const int s = starts ? last_not_above(a.num_seqs, r, [&](int i) { return starts[i]; }) : r;
    const int t = a.lens[s];
    slots[r] = t > 0 ? slot_of(a, s, starts ? t - (starts[s + 1] - r) : t - 1) : -1;
}

// ---- forks

// The first `full` entries of a parent's row for the child as well, every step-th from `first` on.
__device__ __forceinline__ void share_row(const BlocksArgs& a, int parent, int child, int full, int first, int step)
{
    const int32_t* from = a.tables + (size_t)parent * a.max_blocks;
    int32_t* to = a.tables + (size_t)child * a.max_blocks;
    for (int b = first; b < full; b += step) {
        const int id = from[b];
        to[b] = id;
        if (is_block(a, id)) atomicAdd(a.refs + id, 1);
    }
}

__global__ void __launch_bounds__(kPlanThreads)
blocks_fork_kernel(const BlocksArgs a, const int32_t* parents, const int32_t* children, int n, int32_t* copies, int32_t* result,
                   int shares)
{
    __shared__ int sums[kPlanWaves], cut, refused, listed[kListed];
    if (threadIdx.x == 0) refused = 0;
    __syncthreads();
    const uint32_t word = free_word(a, threadIdx.x);        // (asked for with the lengths)
    int* tokens = a.ws.first;
    auto is_seq = [&](int s) { return (uint32_t)s < (uint32_t)a.num_seqs; };
    // (a pair with a negative index is none)
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int p = parents[i], c = children[i];
        tokens[i] = -1;
        if (p < 0 || c < 0) continue;
        if (!is_seq(p) || !is_seq(c) || p == c || a.lens[c] != 0 || a.lens[p] < 0 || blocks_of(a.lens[p]) > a.max_blocks) refused = 1;
        else tokens[i] = a.lens[p];
    }
    __syncthreads();
    // a child named twice: the children's lengths carry the pair's number while all look
    for (int i = threadIdx.x; i < n; i += kPlanThreads)
        if (tokens[i] >= 0) a.lens[children[i]] = -1 - i;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kPlanThreads)
        if (tokens[i] >= 0 && a.lens[children[i]] != -1 - i) refused = 1;
    int need = 0;
    for (int base = 0; base < n; base += kPlanThreads) {
        const int i = base + threadIdx.x;
        int total;
        plan_scan(i < n && tokens[i] > 0 && tokens[i] % kBlock != 0, sums, total);
        need += total;
    }
    __syncthreads();
    int* list = need <= kListed ? listed : a.ws.list;
    const int missing = refused ? -1 : take_blocks(a, word, need, list, sums, &cut);
    if (threadIdx.x == 0) *result = missing;
    __syncthreads();
    int before = 0;
    for (int base = 0; base < n; base += kPlanThreads) {
        const int i = base + threadIdx.x;
        const int t = i < n ? tokens[i] : -1;
        const bool partial = t > 0 && t % kBlock != 0;
        int total;
        const int r = before + plan_scan(partial, sums, total);
        before += total;
        if (i >= n) continue;
        int src = -1, dst = -1;
        if (t >= 0) {
            a.lens[children[i]] = missing == 0 ? t : 0;
            if (partial && missing == 0) {
                const int b = t / kBlock;
                src = a.tables[(size_t)parents[i] * a.max_blocks + b];
                dst = list[r];
                a.tables[(size_t)children[i] * a.max_blocks + b] = dst;
            }
        }
        copies[2 * i] = src;
        copies[2 * i + 1] = dst;
    }
    // (few children: a wavefront each, and no launch behind this one)
    if (shares && missing == 0)
        for (int i = threadIdx.x >> 6; i < n; i += kPlanWaves)
            if (tokens[i] > 0) share_row(a, parents[i], children[i], tokens[i] / kBlock, threadIdx.x & 63, 64);
}

// The full blocks of a parent, shared with the child (blockIdx.y: every so many of them).
__global__ void __launch_bounds__(256)
blocks_share_kernel(const BlocksArgs a, const int32_t* parents, const int32_t* children, const int32_t* result)
{
    const int p = parents[blockIdx.x], c = children[blockIdx.x];
    if (p < 0 || c < 0 || *result != 0) return;
    share_row(a, p, c, a.lens[c] / kBlock, blockIdx.y * 256 + threadIdx.x, gridDim.y * 256);
}

// ---- compaction: of n blocks in use, those numbered n and above move, in order, to the free ones below n

// The new numbers of the blocks that sequence s holds, every step-th entry from `first` on.
__device__ __forceinline__ void renumber_row(const BlocksArgs& a, int s, int used, int first, int step)
{
    const int nb = min(blocks_of(max(a.lens[s], 0)), a.max_blocks);
    int32_t* row = a.tables + (size_t)s * a.max_blocks;
    for (int b = first; b < nb; b += step) {
        const int id = row[b];
        if (!is_block(a, id) || id < used) continue;
        const int to = a.ws.list[id];
        if (is_block(a, to)) row[b] = to;
    }
}

__global__ void __launch_bounds__(kPlanThreads)
blocks_compact_kernel(const BlocksArgs a, int32_t* copies, int32_t* num_copies, int renumbers)
{
    __shared__ int sums[kPlanWaves];
    int used = a.num_blocks;
    for (int base = 0; base < a.words; base += kPlanThreads) {
        int total;
        plan_scan(__builtin_popcount(free_word(a, base + threadIdx.x)), sums, total);
        used -= total;
    }
    int holes = 0, moved = 0;
    for (int base = 0; base < a.words; base += kPlanThreads) {
        const int w = base + threadIdx.x;
        const uint32_t bits = free_word(a, w), front = bits_below(w, used);
        uint32_t to = bits & front, from = ~bits & ~front & bits_below(w, a.num_blocks);
        int total;
        int at = holes + plan_scan(__builtin_popcount(to), sums, total);
        for (; to; to &= to - 1) copies[2 * at++ + 1] = 32 * w + __builtin_ctz(to);
        holes += total;
        at = moved + plan_scan(w < a.words ? __builtin_popcount(from) : 0, sums, total);
        for (; from && w < a.words; from &= from - 1) copies[2 * at++] = 32 * w + __builtin_ctz(from);
        moved += total;
    }
    __syncthreads();
    for (int w = threadIdx.x; w < a.words; w += kPlanThreads) a.free_map[w] = ~bits_below(w, used) & bits_below(w, a.num_blocks);
    for (int k = threadIdx.x; k < moved; k += kPlanThreads) {
        const int src = copies[2 * k], dst = copies[2 * k + 1];
        a.refs[dst] = a.refs[src];
        a.refs[src] = 0;
        a.ws.list[src] = dst;
    }
    if (threadIdx.x == 0) {
        *num_copies = moved;
        *a.ws.used = used;
    }
    if (!renumbers) return;
    __syncthreads();
    for (int s = threadIdx.x >> 6; s < a.num_seqs; s += kPlanWaves) renumber_row(a, s, used, threadIdx.x & 63, 64);
}

__global__ void __launch_bounds__(256)
blocks_renumber_kernel(const BlocksArgs a)
{
    renumber_row(a, blockIdx.x, *a.ws.used, blockIdx.y * 256 + threadIdx.x, gridDim.y * 256);
}

// ---- copying blocks, in all layers of a launch

constexpr int kCopyLayers = 64;

struct CopyLayer {
    uint8_t *k, *v;
    float *ks, *vs;
};
struct CopyArgs {
    const int32_t* copies;
    const int32_t* num_copies;      // NULL: max_copies
    int32_t max_copies, num_blocks, layers;
    uint32_t kv_bytes, scale_bytes; // of a block in one layer
    uint32_t pieces;                // of a block's K and V
    CopyLayer layer[kCopyLayers];
};

typedef uint32_t copy_t __attribute__((ext_vector_type(4), aligned(4)));

constexpr uint32_t kCopyPiece = 16384;         // bytes a workgroup has in flight: 4 loads of 16 a thread

// A piece of a block's K and V in one layer at a time, the scales with the first; all of a piece's loads are asked for
// before its first store.  Bound by HBM where there are enough pieces to fill the chip: 4.85 GB (both ways) of a
// compaction in 16 layers 906 to 928 us, 5.2 to 5.4 TB/s; one block of 8 samples in 40 layers, 21.6 MB, 6.1 us.  (A workgroup per block
// and layer that copied K, then V, 4 KB at a time: 1017 us and 7.1.)
__global__ void __launch_bounds__(256)
blocks_copy_kernel(const CopyArgs a)
{
    const uint32_t n = a.num_copies ? (uint32_t)min(max(*a.num_copies, 0), a.max_copies) : (uint32_t)a.max_copies;
    const uint32_t per_layer = n * a.pieces;                // (the host has seen that it fits)
    for (uint32_t layer = 0, i = blockIdx.x; layer < (uint32_t)a.layers;) {
        if (i >= per_layer) {
            i -= per_layer;
            ++layer;
            continue;
        }
        const uint32_t pair = i / a.pieces, piece = i - pair * a.pieces;
        i += gridDim.x;
        const int src = a.copies[2 * pair], dst = a.copies[2 * pair + 1];
        if ((uint32_t)src >= (uint32_t)a.num_blocks || (uint32_t)dst >= (uint32_t)a.num_blocks) continue;
        const CopyLayer& l = a.layer[layer];
        auto copy_of = [&](uint8_t* k, uint8_t* v, uint32_t bytes, uint32_t at, auto f) {
            if (at < 2 * bytes) {
                uint8_t* pool = at < bytes ? k : v;
                const uint32_t in = at < bytes ? at : at - bytes;
                f(reinterpret_cast<const copy_t*>(pool + (size_t)src * bytes + in), reinterpret_cast<copy_t*>(pool + (size_t)dst * bytes + in));
            }
        };
        copy_t x[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
            copy_of(l.k, l.v, a.kv_bytes, piece * kCopyPiece + 16 * (256 * u + threadIdx.x),
                    [&](const copy_t* from, copy_t*) { x[u] = __builtin_nontemporal_load(from); });
        if (piece == 0 && a.scale_bytes)
            for (uint32_t at = 16 * threadIdx.x; at < 2 * a.scale_bytes; at += 256 * 16)
                copy_of((uint8_t*)l.ks, (uint8_t*)l.vs, a.scale_bytes, at, [&](const copy_t* from, copy_t* to) { *to = *from; });
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
            copy_of(l.k, l.v, a.kv_bytes, piece * kCopyPiece + 16 * (256 * u + threadIdx.x),
                    [&](const copy_t*, copy_t* to) { __builtin_nontemporal_store(x[u], to); });
    }
}

}  // namespace coopt

using namespace coopt;

static BlocksArgs blocks_args(const int32_t* tables, const int32_t* lens, int32_t* refs, uint32_t* free_map, void* workspace,
                              const coopt_shape* sh)
{
    BlocksArgs a{};
    a.tables = const_cast<int32_t*>(tables);
    a.lens = const_cast<int32_t*>(lens);
    a.refs = refs;
    a.free_map = free_map;
    a.ws = blocks_workspace(workspace, sh);
    a.num_seqs = sh->num_seqs;
    a.max_blocks = sh->max_blocks_per_seq;
    a.num_blocks = sh->num_blocks;
    a.words = (int)(((long long)sh->num_blocks + 31) / 32);
    return a;
}

static int check_blocks_workspace(const coopt_shape* sh, const void* workspace, size_t workspace_bytes)
{
    if (!workspace) return COOPT_ERR_NULL;
    if (workspace_bytes < blocks_workspace_bytes(sh) || ((uintptr_t)workspace & 15u) != 0) return COOPT_ERR_WORKSPACE;
    return COOPT_OK;
}

// Workgroups along a row of the table, of 256 entries each.
static unsigned row_workgroups(const coopt_shape* sh)
{
    const int all = (sh->max_blocks_per_seq + 255) / 256;
    return (unsigned)(all < 16 ? all : 16);
}

extern "C" size_t coopt_kv_blocks_workspace_bytes(const coopt_shape* sh)
{
    return check_shape(sh) == COOPT_OK ? blocks_workspace_bytes(sh) : 0;
}

extern "C" int coopt_kv_blocks_init(const int32_t* tables, const int32_t* lens, int32_t* refs, uint32_t* free_map,
                                    const coopt_shape* sh, void* hip_stream)
{
    const int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    if (!refs || !free_map || (sh->num_seqs > 0 && (!tables || !lens))) return COOPT_ERR_NULL;
    hipStream_t stream = (hipStream_t)hip_stream;
    const BlocksArgs a = blocks_args(tables, lens, refs, free_map, nullptr, sh);
    const unsigned wgs = (unsigned)((sh->num_blocks + 255LL) / 256 < 2048 ? (sh->num_blocks + 255LL) / 256 : 2048);
    hipLaunchKernelGGL(blocks_clear_kernel, dim3(wgs), dim3(256), 0, stream, a);
    if (sh->num_seqs > 0) hipLaunchKernelGGL(blocks_count_kernel, dim3((unsigned)sh->num_seqs), dim3(256), 0, stream, a);
    hipLaunchKernelGGL(blocks_map_kernel, dim3(wgs), dim3(256), 0, stream, a);
    return launch_status();
}

extern "C" int coopt_kv_blocks_free(const int32_t* seqs, int32_t num_listed, const int32_t* tables, int32_t* lens, int32_t* refs,
                                    uint32_t* free_map, const coopt_shape* sh, void* hip_stream)
{
    const int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    if (num_listed < 0 || num_listed > (1 << 20)) return COOPT_ERR_SHAPE;
    if (num_listed == 0 || sh->num_seqs == 0) return COOPT_OK;
    if (!seqs || !tables || !lens || !refs || !free_map) return COOPT_ERR_NULL;
    const BlocksArgs a = blocks_args(tables, lens, refs, free_map, nullptr, sh);
    const int threads = sh->max_blocks_per_seq >= 1024 ? 1024 : (sh->max_blocks_per_seq + 63) / 64 * 64;
    hipLaunchKernelGGL(blocks_free_kernel, dim3((unsigned)num_listed), dim3((unsigned)threads), 0, (hipStream_t)hip_stream, a, seqs);
    return launch_status();
}

extern "C" int coopt_kv_blocks_free_outside_window(int32_t* tables, const int32_t* lens, int32_t* refs, uint32_t* free_map,
                                                   int32_t window, int32_t num_sinks, const coopt_shape* sh, void* hip_stream)
{
    const int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    if (window < 1 || num_sinks < 0) return COOPT_ERR_SHAPE;
    if (sh->num_seqs == 0) return COOPT_OK;
    if (!tables || !lens || !refs || !free_map) return COOPT_ERR_NULL;
    const int most = sh->max_blocks_per_seq * kBlock;
    const BlocksArgs a = blocks_args(tables, lens, refs, free_map, nullptr, sh);
    hipLaunchKernelGGL(blocks_free_window_kernel, dim3((unsigned)((sh->num_seqs + 3) / 4)), dim3(256), 0, (hipStream_t)hip_stream, a,
                       window < most ? window : most, num_sinks < most ? num_sinks : most);
    return launch_status();
}

extern "C" int coopt_kv_blocks_reserve(const int32_t* query_start, int32_t num_query_rows, int32_t* tables, int32_t* lens,
                                       int32_t* refs, uint32_t* free_map, int64_t* slot_mapping, int32_t* result, void* workspace,
                                       size_t workspace_bytes, const coopt_shape* sh, void* hip_stream)
{
    int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    if (num_query_rows < 0 || (!query_start && num_query_rows < sh->num_seqs)) return COOPT_ERR_SHAPE;
    if (!result || (sh->num_seqs > 0 && (!tables || !lens || !refs || !free_map || (num_query_rows > 0 && !slot_mapping)))) return COOPT_ERR_NULL;
    st = check_blocks_workspace(sh, workspace, workspace_bytes);
    if (st != COOPT_OK) return st;
    hipStream_t stream = (hipStream_t)hip_stream;
    BlocksArgs a = blocks_args(tables, lens, refs, free_map, workspace, sh);
    if (sh->num_seqs == 0) {                                    // (the map may be NULL, and so may the slots)
        a.words = 0;
        if (!slot_mapping) num_query_rows = 0;
    }
    if (num_query_rows <= 4 * kPlanThreads) {
        hipLaunchKernelGGL(blocks_reserve_kernel<true>, dim3(1), dim3(kPlanThreads), 0, stream, a, query_start, num_query_rows,
                           slot_mapping, result);
    } else {
        hipLaunchKernelGGL(blocks_reserve_kernel<false>, dim3(1), dim3(kPlanThreads), 0, stream, a, query_start, num_query_rows,
                           slot_mapping, result);
        hipLaunchKernelGGL(blocks_slots_kernel, dim3((unsigned)((num_query_rows + 255LL) / 256)), dim3(256), 0, stream, a, query_start,
                           num_query_rows, slot_mapping, result);
    }
    return launch_status();
}

extern "C" int coopt_kv_blocks_fork(const int32_t* parents, const int32_t* children, int32_t num_forks, int32_t* tables, int32_t* lens,
                                    int32_t* refs, uint32_t* free_map, int32_t* copies, int32_t* result, void* workspace,
                                    size_t workspace_bytes, const coopt_shape* sh, void* hip_stream)
{
    int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    if (num_forks < 0 || num_forks > sh->num_seqs) return COOPT_ERR_SHAPE;
    if (!result || (num_forks > 0 && (!parents || !children || !tables || !lens || !refs || !free_map || !copies))) return COOPT_ERR_NULL;
    st = check_blocks_workspace(sh, workspace, workspace_bytes);
    if (st != COOPT_OK) return st;
    hipStream_t stream = (hipStream_t)hip_stream;
    BlocksArgs a = blocks_args(tables, lens, refs, free_map, workspace, sh);
    if (num_forks == 0) a.words = 0;        // (the map may be NULL)
    const bool few = (long long)num_forks * sh->max_blocks_per_seq <= kFewEntries;
    hipLaunchKernelGGL(blocks_fork_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, parents, children, num_forks, copies, result,
                       few ? 1 : 0);
    if (!few)
        hipLaunchKernelGGL(blocks_share_kernel, dim3((unsigned)num_forks, row_workgroups(sh)), dim3(256), 0, stream, a, parents, children,
                           result);
    return launch_status();
}

extern "C" int coopt_kv_blocks_compact(int32_t* tables, const int32_t* lens, int32_t* refs, uint32_t* free_map, int32_t* copies,
                                       int32_t* num_copies, void* workspace, size_t workspace_bytes, const coopt_shape* sh,
                                       void* hip_stream)
{
    int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    if (!refs || !free_map || !num_copies || (sh->num_blocks > 1 && !copies) || (sh->num_seqs > 0 && (!tables || !lens)))
        return COOPT_ERR_NULL;
    st = check_blocks_workspace(sh, workspace, workspace_bytes);
    if (st != COOPT_OK) return st;
    hipStream_t stream = (hipStream_t)hip_stream;
    const BlocksArgs a = blocks_args(tables, lens, refs, free_map, workspace, sh);
    const bool few = (long long)sh->num_seqs * sh->max_blocks_per_seq <= kFewEntries;
    hipLaunchKernelGGL(blocks_compact_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, copies, num_copies, few ? 1 : 0);
    if (!few)
        hipLaunchKernelGGL(blocks_renumber_kernel, dim3((unsigned)sh->num_seqs, row_workgroups(sh)), dim3(256), 0, stream, a);
    return launch_status();
}

extern "C" int coopt_kv_cache_copy_blocks(void* const* k_caches, void* const* v_caches, float* const* k_scales,
                                          float* const* v_scales, int32_t num_layers, const int32_t* copies, int32_t max_copies,
                                          const int32_t* num_copies, const coopt_shape* sh, void* hip_stream)
{
    const int st = check_shape(sh);
    if (st != COOPT_OK) return st;
    const bool scaled = sh->kv_dtype != COOPT_KV_FP16;
    if (num_layers < 0 || max_copies < 0) return COOPT_ERR_SHAPE;
    if (num_layers == 0 || max_copies == 0) return COOPT_OK;
    if (!k_caches || !v_caches || !copies || (scaled && (!k_scales || !v_scales))) return COOPT_ERR_NULL;
    for (int i = 0; i < num_layers; ++i)
        if (!k_caches[i] || !v_caches[i] || (scaled && (!k_scales[i] || !v_scales[i]))) return COOPT_ERR_NULL;
    const long long bytes = (long long)sh->num_kv_heads * kBlock * sh->head_dim * (scaled ? 1 : 2);
    if (2 * bytes > 0x7fffffffLL) return COOPT_ERR_SHAPE;
    for (int l0 = 0; l0 < num_layers; l0 += kCopyLayers) {
        CopyArgs a{};
        a.copies = copies;
        a.num_copies = num_copies;
        a.max_copies = max_copies;
        a.num_blocks = sh->num_blocks;
        a.layers = num_layers - l0 < kCopyLayers ? num_layers - l0 : kCopyLayers;
        a.kv_bytes = (uint32_t)bytes;
        a.scale_bytes = scaled ? (uint32_t)(sh->num_kv_heads * kBlock * 4) : 0;
        for (int i = 0; i < a.layers; ++i)
            a.layer[i] = CopyLayer{(uint8_t*)k_caches[l0 + i], (uint8_t*)v_caches[l0 + i], scaled ? k_scales[l0 + i] : nullptr,
                                   scaled ? v_scales[l0 + i] : nullptr};
        a.pieces = (2 * a.kv_bytes + kCopyPiece - 1) / kCopyPiece;
        const long long per_layer = (long long)max_copies * a.pieces, items = per_layer * a.layers;
        if (per_layer > 0x7fffffffLL) return COOPT_ERR_SHAPE;
        hipLaunchKernelGGL(blocks_copy_kernel, dim3((unsigned)(items < 2048 ? items : 2048)), dim3(256), 0, (hipStream_t)hip_stream, a);
    }
    return launch_status();
}
