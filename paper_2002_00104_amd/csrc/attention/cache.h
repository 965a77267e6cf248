// The paged cache in device code: where a row lies, and which sequence a row of a call belongs to.
#pragma once

#include "../block/rows.h"

namespace pwlq_attention {

using pwlq_block::bf16;
using pwlq_block::f16;
using pwlq_block::v2u;
using pwlq_block::v4f;
using pwlq_block::v4u;
using pwlq_block::v8bf;
using pwlq_block::v8f;
using pwlq_block::v8h;
using pwlq_block::Vec8;

struct Cache {
    char *keys, *values;
    float *key_step, *value_step;
    int pages, heads, shift, D;          // a page holds 2^shift rows of a head
};
struct Batch {
    const int32_t *table, *lengths, *starts;
    int64_t table_stride;
    int S, T, capacity;                  // capacity: rows that a sequence's table has room for
};

inline Cache cache_of(const pwlq_cache &c)
{
    return {(char *)c.keys, (char *)c.values, c.key_step, c.value_step, (int)c.pages, c.heads, __builtin_ctz((unsigned)c.page), c.D};
}
inline Batch batch_of(const pwlq_batch &b, const pwlq_cache &c)
{
    return {b.table, b.lengths, b.starts, b.table_stride, (int)b.S, (int)b.T, (int)(b.table_pages * c.page)};
}

// A sequence's rows in the call, and its length with them.  Whatever the device's arrays hold, rows lie within [0, T) and
// slots within the table.
struct Sequence {
    int start, rows, length;
    __device__ int kept() const { return length - rows; }
};
__device__ inline Sequence sequence(const Batch &b, int s, int start, int end, int length)
{
    Sequence q;
    q.length = min(max(length, 0), b.capacity);
    q.start = min(max(start, 0), b.T);
    q.rows = min(max(end, q.start), b.T) - q.start;
    return q;
}
__device__ inline Sequence sequence(const Batch &b, int s)
{
    return b.starts ? sequence(b, s, b.starts[s], b.starts[s + 1], b.lengths[s]) : sequence(b, s, s, s + 1, b.lengths[s]);
}

// The last s in [0, S) with at(s) <= x for a rising at with at(0) <= x: a wavefront looks at 64 places a turn.
template <typename F> __device__ inline int find_rising(int S, int x, F at)
{
    int lo = 0, n = S;
    while (n > 1) {
        const int step = (n + 63) / 64, i = (int)(threadIdx.x & 63) * step;
        const uint64_t below = __ballot(i < n && at(lo + min(i, n - 1)) <= x);
        const int k = max((int)__popcll(below) - 1, 0);     // it is unsigned: no place is no place before the first
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// A row of the cache, for each of its heads: page and row in it.  page is -1 where there is none.
struct Place { int page, row; };
__device__ inline Place place(const Cache &c, const Batch &b, int s, int slot)
{
    Place p = {-1, slot & ((1 << c.shift) - 1)};
    if (slot >= 0 && slot < b.capacity) {
        const int page = b.table[s * b.table_stride + (slot >> c.shift)];
        if ((unsigned)page < (unsigned)c.pages) p.page = page;
    }
    return p;
}
// Its number among all rows of all heads: an element's place is that times D, a step's is that itself.
__device__ inline int64_t row_number(const Cache &c, Place p, int head) { return (((int64_t)p.page * c.heads + head) << c.shift) + p.row; }

} // namespace pwlq_attention
