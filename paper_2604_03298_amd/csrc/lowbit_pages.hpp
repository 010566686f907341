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

constexpr uint32_t MAX_TOKENS = 1u << 24;       // of a call: a workgroup of 256 each is what a launch holds
constexpr int32_t MAX_SEQUENCE = 1 << 30;       // tokens: positions and the ends of pages stay below 2^31

// A sequence's part of a call: tokens start ... start + count - 1 of the call end a sequence of `length` tokens.
struct Sequence {
    uint32_t start, count;
    int32_t length;
    bool good;
};
__device__ __forceinline__ bool in_order(const Pages &c, int32_t start, int32_t next) { return start >= 0 && start <= next && (uint32_t)next <= c.n_tokens; }
__device__ __forceinline__ Sequence sequence_from(const Pages &c, int32_t s, int32_t e, int32_t n, int32_t most)
{
    const int64_t room = (int64_t)c.table_stride << c.log_page;
    const bool good = in_order(c, s, e) && n >= 0 && n <= most && (int64_t)n <= room;
    return {(uint32_t)s, (uint32_t)(e - s), n, good};
}
__device__ __forceinline__ Sequence sequence_of(const Pages &c, uint32_t b, int32_t most)
{
    return sequence_from(c, c.starts[b], c.starts[b + 1], c.lengths[b], most);
}

// Work is handed out by page.  A sequence with t tokens in the call touches at most (t - 1) div P + 2 pages, so sequence b gets the
// items from starts[b] div P + 2 b on: these ranges do not overlap, and starts[batch] div P + 2 batch items are enough for
// all, whatever the lengths, which only the device knows.  Every wave finds its item's sequence by itself: the starts ascend, so
// it is the last one whose range begins at or before the item.  What is known of the sequence comes along with the search.  Sequences whose
// starts are out of order have no items, wherever their starts point to: the workgroup of the first item looks at all of them and tells of such.
struct Found {
    int32_t b;                  // -1: none
    uint32_t first;             // its first item
    Sequence s;
};
__device__ __forceinline__ Found sequence_of_item(const Pages &c, uint32_t item)
{
    const uint32_t lane = threadIdx.x & 63;
    Found f{};
    f.b = -1;
    for (uint32_t b = 0; b < c.batch; b += 64) {
        const uint32_t i = b + lane < c.batch ? b + lane : c.batch - 1;
        const int32_t start = c.starts[i], next = c.starts[i + 1], length = c.lengths[i];
        const bool there = b + lane < c.batch, good = in_order(c, start, next);
        const uint64_t some = __ballot(there && good);
        const uint64_t before = __ballot(there && good && (uint32_t)(start >> c.log_page) + 2 * i <= item);
        if (item == 0 && __any(there && !good)) complain(c);
        if (before) {
            const int last = 63 - __builtin_clzll(before);
            f.b = (int32_t)b + last;
            const int32_t s = __builtin_amdgcn_readlane(start, last);
            f.first = (uint32_t)(s >> c.log_page) + 2 * (uint32_t)f.b;
            f.s = sequence_from(c, s, __builtin_amdgcn_readlane(next, last), __builtin_amdgcn_readlane(length, last), MAX_SEQUENCE);
        }
        if (item != 0 && before != some) break;              // the later ones' ranges begin further on
    }
    return f;
}

}  // namespace lowbit
}  // namespace enec
