// The pages of a batch of sequences, as the kernels of the cache and of its attention see them.
#pragma once

#include "lowbit.hpp"

namespace enec {
namespace lowbit {

struct Pages {
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t *table, *starts, *lengths;
    uint32_t *status;
    uint32_t n_pages, log_page, heads, head_dim, table_stride, batch, n_tokens;
};

constexpr uint32_t STATUS_ARG = 1;      // ENEC_E_ARG

__device__ __forceinline__ void complain(const Pages &c)
{
    if (c.status) *reinterpret_cast<volatile uint32_t *>(c.status) = STATUS_ARG;
}

constexpr int32_t MAX_SEQUENCE = 1 << 30;       // tokens: positions and the ends of pages stay below 2^31

// A sequence's part of a call: tokens start ... start + count - 1 of the call end a sequence of `length` tokens.
struct Sequence {
    uint32_t start, count;
    int32_t length;
    bool good;
};
__device__ __forceinline__ Sequence sequence_of(const Pages &c, uint32_t b, int32_t most)
{
    const int32_t s = c.starts[b], e = c.starts[b + 1], n = c.lengths[b];
    const int64_t room = (int64_t)c.table_stride << c.log_page;
    const bool good = s >= 0 && e >= s && (uint32_t)e <= c.n_tokens && n >= 0 && n <= most && (int64_t)n <= room;
    return {(uint32_t)s, (uint32_t)(e - s), n, good};
}

// Work is handed out by page.  A sequence with t tokens in the call touches at most (t - 1) div P + 2 pages, so sequence b gets the
// items from starts[b] div P + 2 b on: these ranges do not overlap, and starts[batch] div P + 2 batch items are enough for
// all, whatever the lengths, which only the device knows.  Every wave finds its item's sequence by itself: the starts ascend, so
// it is the number of sequences whose range begins at or before the item.
__device__ __forceinline__ int32_t sequence_of_item(const Pages &c, uint32_t item, uint32_t &first)
{
    uint32_t n = 0;
    const uint32_t lane = threadIdx.x & 63;
    for (uint32_t b = 0; b < c.batch; b += 64) {
        const uint32_t i = b + lane;
        const bool before = i < c.batch && (int64_t)(c.starts[i] >> c.log_page) + 2 * (int64_t)i <= (int64_t)item;
        n += (uint32_t)__popcll(__ballot(before));
    }
    if (n == 0) return -1;
    first = (uint32_t)(c.starts[n - 1] >> c.log_page) + 2 * (n - 1);
    return (int32_t)n - 1;
}

}  // namespace lowbit
}  // namespace enec
