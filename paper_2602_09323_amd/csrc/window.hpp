// Attention through a sliding window: the token at position p sees the tokens j <= p with
// j > p - size (the last `size` ones, itself included) or j < sinks (the sequence's first).
//
// Seen from the tokens at positions first + size - 1 and after, a sequence is its sinks' blocks and the
// blocks from token `first` on.  WindowView renumbers these as if nothing lay between them, so that a
// kernel which streams a whole context streams this one: it has `t` tokens, its block b is block block(b)
// of the table, and of its tokens only the gap [lo, hi) is hidden from all -- the rest of the last
// sinks' block and what the block of `first` holds in front of it, fewer than 31 tokens, so that two
// blocks (32 tokens) always hold one that is seen.  Blocks that are left out are never read, nor are their
// table entries: they may be anything.
//
// (Plain C++ but for the two function qualifiers: a host program can include it.)
#pragma once

#include <stdint.h>

#include "coopt_attn.h"

namespace coopt {

struct Window {
    int32_t size, sinks;      // >= 1; >= 0
};

struct WindowView {
    static constexpr int kB = 16;      // tokens per block
    int t;            // tokens, those of blocks left out not counted
    int lead, skip;   // blocks in front of the ones left out, and how many these are
    int lo, hi;       // hidden tokens (none where hi <= lo)

    // Of a sequence of `tokens`, what the tokens whose windows begin at `first` or later see.
    __device__ __forceinline__ WindowView(const Window& w, int tokens, int first)
    {
        const int begin = first > 0 ? first : 0;
        lead = (w.sinks + kB - 1) / kB;
        skip = begin / kB > lead ? begin / kB - lead : 0;
        t = tokens - skip * kB;
        lo = w.sinks;
        hi = begin - skip * kB;
    }
    // ... what its last token sees.
    __device__ __forceinline__ WindowView(const Window& w, int tokens) : WindowView(w, tokens, tokens - w.size) {}
    __device__ __forceinline__ int block(int b) const { return b < lead ? b : b + skip; }
};

// Arguments of the entry points; behind check_shape.
inline int check_window(int window, int num_sinks) { return window >= 1 && num_sinks >= 0 ? COOPT_OK : COOPT_ERR_SHAPE; }

// Both clamped to what a table holds (2^28 tokens at most: no sum overflows).
inline Window window_of(const coopt_shape* sh, int window, int num_sinks)
{
    const int most = sh->max_blocks_per_seq * sh->block_size;
    return Window{window < most ? window : most, num_sinks < most ? num_sinks : most};
}

// The tokens that a row sees at most.
inline long long window_row_tokens(const coopt_shape* sh, const Window& w)
{
    const long long most = (long long)sh->max_blocks_per_seq * sh->block_size, seen = (long long)w.size + w.sinks;
    return seen < most ? seen : most;
}

// The shape with a table as wide as the most blocks that a view over `rows` neighbouring tokens' windows has.
inline coopt_shape window_shape(const coopt_shape* sh, const Window& w, int rows = 1)
{
    coopt_shape s = *sh;
    const long long tokens = (long long)w.size + rows - 1;
    const long long blocks = (w.sinks + 15) / 16 + (tokens + 14) / 16 + 1;
    if (blocks < s.max_blocks_per_seq) s.max_blocks_per_seq = (int)blocks;
    return s;
}

}  // namespace coopt
