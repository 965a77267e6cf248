// pwlq_attend: which kernel, how a call is cut, and the join of the parts of an item.
#include "attend.h"

namespace pwlq_attention {

// attend_bf16.hip and its like, one for each pair of types; D: channels that the kernel is made for; rows of a tile
template <typename T, typename C> void attend_launch(const Attend &a, int D, int rows, unsigned grid, hipStream_t stream);
extern template PWLQ_INTERNAL void attend_launch<bf16, bf16>(const Attend &, int, int, unsigned, hipStream_t);
extern template PWLQ_INTERNAL void attend_launch<bf16, int8_t>(const Attend &, int, int, unsigned, hipStream_t);
extern template PWLQ_INTERNAL void attend_launch<f16, f16>(const Attend &, int, int, unsigned, hipStream_t);
extern template PWLQ_INTERNAL void attend_launch<f16, int8_t>(const Attend &, int, int, unsigned, hipStream_t);

namespace {

// The parts of an item that workgroups left in the workspace: DP / 4 lanes a group, a workgroup for ROWS rows, each of which has a group or several;
// these take its parts in turn, each in the order of the keys, and the first adds up what they have, in their order.  3.5 us (a launch) for a token, 6 for
// one in 512 parts, 8 for 37 MB of sums of 228 items.
template <typename T, int DP, int ROWS> __global__ __launch_bounds__(256) void k_attend_join(const Attend a, int rows)
{
    constexpr int kLanes = DP / 4, kGroups = 256 / kLanes, kEach = kGroups > ROWS ? kGroups / ROWS : 1;
    __shared__ v4f sums[kGroups][kLanes];
    __shared__ float2 tops[kGroups];
    const Stretch t = a.stretches[blockIdx.x];
    // the parts with its first unit and its last
    const int part = *a.part, n = t.units + kSetup, x = t.begin * a.c.heads + blockIdx.y * n;
    if (t.units == 0 || t.first + (int)blockIdx.z * ROWS >= t.rows) return;
    const int first = (uint32_t)(x + kSetup) / (uint32_t)part, last = (uint32_t)(x + n - 1) / (uint32_t)part;
    if (first == last) return;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes, turn = group % kEach, d = 4 * lane;
#pragma unroll
    for (int r = 0; r < ROWS; r += kGroups / kEach) {
        const int of = blockIdx.z * ROWS + r + group / kEach, row = t.first + of;
        v4f v = {};
        float top = -INFINITY, total = 0.0f;
        auto add = [&](float2 o, v4f s) {
            const float most = fmaxf(top, o.x);
            const float old = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - most);
            const float now = o.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(o.x - most);
            v = v * old + s * now;
            total = total * old + o.y * now;
            top = most;
        };
        if (row < t.rows) {
#pragma unroll 4
            for (int w = first + turn; w <= last; w += kEach) {
                const int64_t at = (int64_t)(2 * w + (x > w * part)) * rows + of;
                add(a.top_sum[at], *(const v4f *)(a.sums + at * DP + d));
            }
        }
        if constexpr (kEach > 1) {
            sums[group][lane] = v;
            if (lane == 0) tops[group] = make_float2(top, total);
            __syncthreads();
            if (turn == 0)
                for (int g = 1; g < kEach; ++g) add(tops[group + g], sums[group + g][lane]);
        }
        if (turn != 0 || row >= t.rows || d >= a.c.D) continue;
        const int j = by_group(a, row), h = blockIdx.y * a.group + row - j * a.group;
        store4<T>(a.out + ((t.start + j) * a.out_stride + h * a.out_head + d) * 2, total == 0.0f ? v4f{} : v * (1.0f / total));
    }
}


// Units of keys up to which an item is a workgroup's whole: cutting the line costs 4 to 6 us, in the join's launch and in laying the line out, so a
// single item is cut where its units take longer than that; with more items the parts are no shorter than items are, and only the limit on
// what one long sequence among short ones may cost holds (10 units, or 24 of many rows).  Whole and cut, in us, 8 heads of the cache of 128 channels, bfloat16:
//   tokens of 1, 8 and 48 sequences   301 rows 9.2, 10.0; 9.4, 11.4; 15.7, 19.6      701 rows 12.4, 10.6; 12.6, 14.1; 25.7, 30.4
//   64 rows of 1, 8 and 48            264 rows 16.0, 18.5; 16.9, 26.1; 41.4, 41.7    764 rows 23.9, 19.9; 26.1, 32.4; 65.1, 65.1
// Tokens cost less a unit in 64 channels (7.1, 9.3 for 301 rows of 1) and more in 256 (16.7, 14.0), many rows more with 8-bit caches (19.3, 21.3 and 32.9,
// 21.9) and in 256 channels, where a launch of several workgroups for each CU is slower than a cut one (768 items of 164 rows 84.8, 70.7).
int64_t whole_units(int rows, int channels, bool codes, int64_t items)
{
    if (rows == 128) {
        if (channels == 256 && items > 256) return 0;
        const int64_t most = items < 144 ? 6 + items / 8 : 24;
        return codes || channels == 256 ? most / 2 : most;
    }
    const int64_t most = (items < 384 ? 4 + items / 64 : 10) - (rows == 32);
    return channels == 64 ? most * 3 / 2 : channels == 256 ? most / 2 : most;
}

struct Shape { int rows, channels, unit, tiles, each, parts, least; size_t part, stretches, top_sum, sums, bytes; };

Shape shape_of(const pwlq_attend_args &g)
{
    Shape s = {};
    // longest and window may be any numbers: no more is made of them than there are rows and slots
    const int64_t group = g.q_heads / g.cache.heads, longest = !g.batch.starts ? 1 : g.longest && g.longest < g.batch.T ? g.longest : g.batch.T;
    s.channels = g.cache.D <= 64 ? 64 : g.cache.D <= 128 ? 128 : 256;
    // A tile for all rows of a sequence, so that its keys are read once.  16 sequences of 4000 rows, trees of 20 rows, in tiles of 16, 32 and 128:
    // 93, 62 and 64 us, 57, 53 and 67 with an 8-bit cache; of 48 rows 130, 67 and 69, 77, 76 and 73.
    const int64_t rows = longest * group;
    s.rows = rows <= 16 ? 16 : rows <= 32 && s.channels != 256 ? 32 : 128;
    s.unit = s.rows < 128 ? 128 : s.channels == 256 ? 32 : 64;
    s.each = (int)((group + s.rows - 1) / s.rows);
    const int64_t tiles = g.batch.starts ? g.batch.T * group / s.rows + g.batch.S : g.batch.S * s.each;
    s.tiles = (int)tiles;
    s.least = s.rows < 128 ? 1 : 4;
    // what an item may see: the table, or the window of its first row to its last
    const int64_t table = g.batch.table_pages * g.cache.page, window = (g.window < table ? g.window : table) + s.rows / group + 1;
    const bool windowed = g.window > 0 && g.window < table && !g.prefix && window < table;
    const int64_t units = windowed ? (window + s.unit - 1) / s.unit + 1 : (table + s.unit - 1) / s.unit, items = tiles * g.cache.heads;
    // Tiles of one sequence run beside each other and share its keys in the L2s as whole items, and as parts they are anywhere: where there are
    // many, and items enough to fill the chip, they stay whole (32 heads over 8 of 128 channels, whole and cut: a prompt of 2048 rows 59 and 74 us, 1024
    // items of 4096 156 and 184, after 4000 in 8 bits 511 and 565; of 256 channels 133 and 243).  Where they are few, parts are the better balance
    // (100 sequences of 1128, the last 128 of one head, in 8 bits 233 and 143, in 16 167 both; 12 of 5160, the last 160 of 4 heads, in 8 bits 371 and 251).
    const bool enough = (s.rows == 128 && items >= (rows >= 8 * 128 ? 512 : 4096)) || units <= whole_units(s.rows, s.channels, g.cache.type == PWLQ_I8, items);
    if (tiles <= kMostTiles && g.batch.S <= kMostTiles && items * (units + kSetup + 1) < 1LL << 30 && !enough) {
        const int64_t all = items * ((units > 1 ? units : 1) + kSetup);
        const int64_t parts = (all + s.least - 1) / s.least;
        const int most = s.channels == 256 || (s.rows == 32 && s.channels == 128) ? 256 : 512;    // what the chip holds at once
        s.parts = (int)(parts < most ? parts : most);
    }
    auto place = [&](size_t bytes) {
        const size_t at = s.bytes;
        s.bytes = (s.bytes + bytes + 255) & ~(size_t)255;
        return at;
    };
    if (s.parts) {
        s.part = place(8);
        s.stretches = place(sizeof(Stretch) * (size_t)s.tiles);
        s.top_sum = place(8 * 2 * (size_t)s.parts * s.rows);
        s.sums = place(4 * 2 * (size_t)s.parts * s.rows * s.channels);
    }
    return s;
}

} // namespace

size_t attend_workspace(const pwlq_attend_args &a) { return shape_of(a).bytes; }

void attend(const pwlq_attend_args &g, void *workspace, hipStream_t stream)
{
    const Shape s = shape_of(g);
    Attend a = {};
    a.c = cache_of(g.cache);
    a.b = batch_of(g.batch, g.cache);
    a.q = (const char *)g.q.data;
    a.out = (char *)g.out.data;
    a.q_stride = g.q.stride, a.q_head = g.q.head_stride;
    a.out_stride = g.out.stride, a.out_head = g.out.head_stride;
    a.group = g.q_heads / g.cache.heads;
    a.per_group = ((1ULL << 40) + a.group - 1) / a.group;
    a.scale = g.scale;
    a.cap = g.cap;
    a.slopes = g.slopes;
    a.window = (int)(g.window < a.b.capacity ? g.window : 0);      // one as long as the table holds nothing back
    a.prefix = g.prefix;
    a.tree = g.tree;
    a.tree_words = (int)g.tree_words;
    a.tiles = s.tiles;
    a.each = s.each;
    a.parts = s.parts;
    a.least = s.least;
    a.alone = s.rows < 128 ? 1 : 8;
    char *const w = (char *)workspace;
    a.part = (int *)(w + s.part);
    a.stretches = (Stretch *)(w + s.stretches);
    a.top_sum = (float2 *)(w + s.top_sum);
    a.sums = (float *)(w + s.sums);
    const int64_t items = (int64_t)s.tiles * a.c.heads;
    const unsigned grid = s.parts ? (unsigned)s.parts : (unsigned)(items < 1 << 22 ? items : 1 << 22);
    const bool codes = g.cache.type == PWLQ_I8;
    if (g.q.type == PWLQ_BF16) {
        if (codes) attend_launch<bf16, int8_t>(a, s.channels, s.rows, grid, stream);
        else attend_launch<bf16, bf16>(a, s.channels, s.rows, grid, stream);
    } else {
        if (codes) attend_launch<f16, int8_t>(a, s.channels, s.rows, grid, stream);
        else attend_launch<f16, f16>(a, s.channels, s.rows, grid, stream);
    }
    if (s.parts < 2) return;
#define PWLQ_JOIN_ROWS(T, DP, ROWS)                                                                                  \
    k_attend_join<T, DP, ROWS><<<dim3((unsigned)s.tiles, (unsigned)a.c.heads, (unsigned)(s.rows / (ROWS))), 256, 0, stream>>>(a, s.rows)
#define PWLQ_JOIN(T)                                                                         \
    do {                                                                                     \
        if (s.rows < 128 && s.parts >= 16 * s.tiles * a.c.heads) {                           \
            if (s.channels == 64) PWLQ_JOIN_ROWS(T, 64, 1);                                  \
            else if (s.channels == 128) PWLQ_JOIN_ROWS(T, 128, 1);                           \
            else PWLQ_JOIN_ROWS(T, 256, 1);                                                  \
        } else if (s.rows < 128) {                                                           \
            if (s.channels == 64) PWLQ_JOIN_ROWS(T, 64, 2);                                  \
            else if (s.channels == 128) PWLQ_JOIN_ROWS(T, 128, 2);                           \
            else PWLQ_JOIN_ROWS(T, 256, 2);                                                  \
        } else {                                                                             \
            if (s.channels == 64) PWLQ_JOIN_ROWS(T, 64, 8);                                 \
            else if (s.channels == 128) PWLQ_JOIN_ROWS(T, 128, 8);                          \
            else PWLQ_JOIN_ROWS(T, 256, 4);                                                 \
        }                                                                                    \
    } while (0)
    if (g.q.type == PWLQ_BF16) PWLQ_JOIN(bf16);
    else PWLQ_JOIN(f16);
#undef PWLQ_JOIN
#undef PWLQ_JOIN_ROWS
}

} // namespace pwlq_attention
