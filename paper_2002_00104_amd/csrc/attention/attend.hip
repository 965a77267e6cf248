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

// The parts of an item that workgroups left in the workspace, in the order of the keys: a workgroup for 16 rows of an item.
template <typename T, int DP> __global__ __launch_bounds__(256) void k_attend_join(const Attend a, int rows)
{
    const int u = blockIdx.x, head = blockIdx.y;
    const int64_t n = a.begin[u + 1] - a.begin[u];
    if (n == 0) return;
    const int64_t part = (int64_t)*a.part, x = (int64_t)a.begin[u] * a.c.heads + head * n, first = x / part, last = (x + n - 1) / part;
    if (first == last) return;
    const Tile t = tile(a, u, rows);
    for (int i = threadIdx.x + blockIdx.z * (16 * DP / 4); i < (int)(blockIdx.z + 1) * (16 * DP / 4); i += 256) {
        const int of = i / (DP / 4), d = i % (DP / 4) * 4, row = t.first + of;
        if (row >= t.rows || d >= a.c.D) continue;
        v4f v = {};
        float top = -INFINITY, total = 0.0f;
        for (int64_t w = first; w <= last; ++w) {
            const int64_t at = (2 * w + (x > w * part)) * rows + of;
            const float2 o = a.top_sum[at];
            const v4f s = *(const v4f *)(a.sums + at * DP + d);
            const float most = fmaxf(top, o.x);
            const float old = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - most);
            const float now = o.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(o.x - most);
            v = v * old + s * now;
            total = total * old + o.y * now;
            top = most;
        }
        const int j = row / a.group, h = head * a.group + row - j * a.group;
        store4<T>(a.out + ((t.q.start + j) * a.out_stride + h * a.out_head + d) * 2, total == 0.0f ? v4f{} : v * (1.0f / total));
    }
}

constexpr int kParts = 512;              // two workgroups for each CU

struct Shape { int rows, channels, unit, tiles, each, parts, least; size_t part, begin, top_sum, sums, bytes; };

Shape shape_of(const pwlq_attend_args &g)
{
    Shape s = {};
    const int64_t group = g.q_heads / g.cache.heads, longest = !g.batch.starts ? 1 : g.longest ? g.longest : g.batch.T;
    s.channels = g.cache.D <= 64 ? 64 : g.cache.D <= 128 ? 128 : 256;
    s.rows = longest * group <= 16 ? 16 : longest * group <= 32 ? 32 : 128;
    s.unit = s.rows < 128 ? 128 : s.channels == 256 ? 32 : 64;
    s.each = (int)((group + s.rows - 1) / s.rows);
    const int64_t tiles = g.batch.starts ? g.batch.T * group / s.rows + g.batch.S : g.batch.S * s.each;
    s.tiles = (int)tiles;
    s.least = s.rows < 128 ? 1 : 4;
    const int64_t units = (g.batch.table_pages * g.cache.page + s.unit - 1) / s.unit, items = tiles * g.cache.heads;
    const bool enough = s.rows == 128 && items >= 1024;
    if (tiles <= kMostTiles && g.batch.S <= kMostTiles && tiles * units < 1LL << 31 && !enough) {
        const int64_t all = items * (units > 1 ? units : 1);
        const int64_t parts = (all + s.least - 1) / s.least;
        s.parts = (int)(parts < kParts ? parts : kParts);
    }
    auto place = [&](size_t bytes) {
        const size_t at = s.bytes;
        s.bytes = (s.bytes + bytes + 255) & ~(size_t)255;
        return at;
    };
    if (s.parts) {
        s.part = place(8);
        s.begin = place(4 * (size_t)(s.tiles + 1));
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
    char *const w = (char *)workspace;
    a.part = (uint64_t *)(w + s.part);
    a.begin = (uint32_t *)(w + s.begin);
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
    const dim3 join((unsigned)s.tiles, (unsigned)a.c.heads, (unsigned)(s.rows / 16));
#define PWLQ_JOIN(T)                                                                         \
    do {                                                                                     \
        if (s.channels == 64) k_attend_join<T, 64><<<join, 256, 0, stream>>>(a, s.rows);     \
        else if (s.channels == 128) k_attend_join<T, 128><<<join, 256, 0, stream>>>(a, s.rows); \
        else k_attend_join<T, 256><<<join, 256, 0, stream>>>(a, s.rows);                     \
    } while (0)
    if (g.q.type == PWLQ_BF16) PWLQ_JOIN(bf16);
    else PWLQ_JOIN(f16);
#undef PWLQ_JOIN
}

} // namespace pwlq_attention
