// k_append: new rows into the paged cache, queries and keys turned by their positions.  k_read: rows of the cache.
//
//   angle = position * frequency,  (a, b) -> (a cos - b sin, b cos + a sin) for each pair of channels
//   code = rne(x * (127/a)),  step = a/127,  a the largest magnitude of a row of a head (8-bit caches)
// Both are bound by memory: each element is read once and written once, and with few rows by latency.  3795 rows of 32 + 16 heads of 128
// channels into an 8-bit cache 21.3 us (86 MB, 4.0 TB/s), read back 7.9 (23 MB); a single row 3.3 us, which is a launch.
//
// A workgroup takes one row of the call or several.  Their angles come first, one to a thread: binary64, reduced to a fraction
// of a turn there, since position * frequency has no fraction left in binary32 for far positions.  All heads of a row share them,
// through LDS.  A head of a row is then one group of lanes with eight neighbouring channels each.
#include "launch.h"
#include "cache.h"

namespace pwlq_attention {
namespace {

using pwlq_block::load8;
using pwlq_block::store8;

constexpr int kRows = 4;                // rows of the call in a workgroup, at most
constexpr int kMostPairs = 128;

struct Append {
    Cache c;
    Batch b;
    const char *q, *k, *v;
    char *q_out;
    int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head, out_stride, out_head;
    int q_heads, pairs, interleaved, rows, heads_each;     // rows of the call and heads (of q, k and v together) a workgroup takes
    const int32_t *positions;
    const float *frequencies;
};

struct Row { int number; Place place; };                   // of the call (-1: none), and where it is in the cache

// The call's row t: one wavefront.
__device__ inline Row row_of(const Cache &c, const Batch &b, int t, int &slot)
{
    Row r = {-1, {-1, 0}};
    slot = 0;
    if (t >= b.T) return r;
    const int s = b.starts ? find_rising(b.S, t, [&](int i) { return b.starts[i]; }) : t;
    const Sequence q = sequence(b, s);
    if (t < q.start || t - q.start >= q.rows) return r;
    r.number = t;
    slot = q.kept() + (t - q.start);
    r.place = place(c, b, s, slot);
    return r;
}

// Sine and cosine of angle = position * frequency.  The turns' whole part goes in binary64; what is left is exact to 2^-53 of the
// angle, and the functions of half turns add no reduction of their own.
__device__ inline float2 turn(int position, float frequency)
{
    const double turns = (double)position * (double)frequency * 0.15915494309189533577;
    const float part = (float)(2.0 * (turns - __builtin_rint(turns)));
    return make_float2(cospif(part), sinpif(part));
}

// LANES: lanes of a head, eight channels each.  C: element type of the cache.
template <typename T, typename C, int LANES>
__global__ __launch_bounds__(256) void k_append(Append a)
{
    __shared__ float2 turns[kRows][kMostPairs];
    __shared__ Row rows[kRows];
    __shared__ int slots[kRows];
    const int wave = threadIdx.x >> 6, first = blockIdx.x * a.rows;
    if (wave < a.rows) {
        int slot;
        const Row r = row_of(a.c, a.b, first + wave, slot);
        if ((threadIdx.x & 63) == 0) {
            rows[wave] = r;
            slots[wave] = slot;
        }
    }
    __syncthreads();
    if (a.pairs) {
        for (int i = threadIdx.x; i < a.rows * a.pairs; i += 256) {
            const int r = i / a.pairs, p = i - r * a.pairs;
            if (rows[r].number >= 0) turns[r][p] = turn(a.positions ? a.positions[rows[r].number] : slots[r], a.frequencies[p]);
        }
        __syncthreads();
    }
    const int D = a.c.D, lane = threadIdx.x % LANES, d = 8 * lane;
    const int all = a.q_heads + 2 * a.c.heads, from = blockIdx.y * a.heads_each, to = min(from + a.heads_each, all);
    for (int i = threadIdx.x / LANES; i < a.rows * (to - from); i += 256 / LANES) {
        const int r = i / (to - from), h = from + i - r * (to - from);
        const Row row = rows[r];
        if (row.number < 0) continue;                       // the same for all lanes of the head
        const bool query = h < a.q_heads, key = !query && h < a.q_heads + a.c.heads;
        const int head = query ? h : key ? h - a.q_heads : h - a.q_heads - a.c.heads;
        if (!query && row.place.page < 0) continue;
        const T *in = query ? (const T *)a.q + row.number * a.q_stride + head * a.q_head
                      : key ? (const T *)a.k + row.number * a.k_stride + head * a.k_head
                            : (const T *)a.v + row.number * a.v_stride + head * a.v_head;
        v8f x = {};
        if (d < D) x = pwlq_block::widen(load8<T>(in + d));
        if ((query || key) && d < 2 * a.pairs) {
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 t = turns[r][d / 2 + j];
                    const float u = x[2 * j] * t.x - x[2 * j + 1] * t.y, w = x[2 * j + 1] * t.x + x[2 * j] * t.y;
                    x[2 * j] = u;
                    x[2 * j + 1] = w;
                }
            } else {
                // a multiple of eight pairs: the others' eight channels are a vector too
                const bool upper = d >= a.pairs;
                const int p = upper ? d - a.pairs : d;
                const v8f y = pwlq_block::widen(load8<T>(in + (upper ? p : d + a.pairs)));
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float2 t = turns[r][p + j];
                    x[j] = upper ? x[j] * t.x + y[j] * t.y : x[j] * t.x - y[j] * t.y;
                }
            }
        }
        if (query) {
            if (d < D) store8<T>((T *)a.q_out + row.number * a.out_stride + head * a.out_head + d, __builtin_convertvector(x, typename Vec8<T>::type));
            continue;
        }
        const int64_t n = row_number(a.c, row.place, head);
        char *const out = key ? a.c.keys : a.c.values;
        if constexpr (sizeof(C) == 1) {
            const float v[8] = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
            uint32_t top = pwlq_block::largest(v);
#pragma unroll
            for (int k = 1; k < LANES; k *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, k));
            const pwlq_block::Step s = pwlq_block::step_of(top);
            v2u codes = {0u, 0u};
            if (s.factor != 0.0f) codes = v2u{pwlq_block::four_codes(v, s.factor), pwlq_block::four_codes(v + 4, s.factor)};
            if (d < D) store8<int8_t>((int8_t *)out + n * D + d, codes);
            if (lane == 0) (key ? a.c.key_step : a.c.value_step)[n] = s.step;
        } else {
            if (d < D) store8<T>((T *)out + n * D + d, __builtin_convertvector(x, typename Vec8<T>::type));
        }
    }
}

struct Read {
    Cache c;
    Batch b;
    char *k, *v;
    int64_t k_stride, k_head, v_stride, v_head;
    int rows;                                              // of the call a workgroup takes
};

template <typename T, typename C, int LANES>
__global__ __launch_bounds__(256) void k_read(Read a)
{
    __shared__ Row rows[kRows];
    const int wave = threadIdx.x >> 6, D = a.c.D, lane = threadIdx.x % LANES, d = 8 * lane;
    if (wave < a.rows) {
        int slot;
        const Row r = row_of(a.c, a.b, blockIdx.x * a.rows + wave, slot);
        if ((threadIdx.x & 63) == 0) rows[wave] = r;
    }
    __syncthreads();
    for (int i = threadIdx.x / LANES; i < a.rows * 2 * a.c.heads; i += 256 / LANES) {
        const int of = i / (2 * a.c.heads), h = i - of * 2 * a.c.heads;
        const Row row = rows[of];
        const bool key = h < a.c.heads;
        const int head = key ? h : h - a.c.heads;
        char *const out = key ? a.k : a.v;
        if (row.number < 0 || !out || d >= D) continue;
        v8f x = {};
        if (row.place.page >= 0) {
            const int64_t n = row_number(a.c, row.place, head);
            x = pwlq_block::widen(load8<C>((const C *)(key ? a.c.keys : a.c.values) + n * D + d));
            if constexpr (sizeof(C) == 1) {
                const float step = (key ? a.c.key_step : a.c.value_step)[n];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= step;
            }
        }
        T *const to = (T *)out + row.number * (key ? a.k_stride : a.v_stride) + head * (key ? a.k_head : a.v_head) + d;
        store8<T>(to, __builtin_convertvector(x, typename Vec8<T>::type));
    }
}

#define PWLQ_LANES(KERNEL, T, C, D, ...)                                   \
    do {                                                                   \
        if ((D) <= 16) KERNEL<T, C, 2> __VA_ARGS__;                        \
        else if ((D) <= 32) KERNEL<T, C, 4> __VA_ARGS__;                   \
        else if ((D) <= 64) KERNEL<T, C, 8> __VA_ARGS__;                   \
        else if ((D) <= 128) KERNEL<T, C, 16> __VA_ARGS__;                 \
        else KERNEL<T, C, 32> __VA_ARGS__;                                 \
    } while (0)
#define PWLQ_TYPES(KERNEL, type, cache_type, D, ...)                                        \
    do {                                                                                    \
        if ((type) == PWLQ_BF16) {                                                          \
            if ((cache_type) == PWLQ_I8) PWLQ_LANES(KERNEL, bf16, int8_t, D, __VA_ARGS__);  \
            else PWLQ_LANES(KERNEL, bf16, bf16, D, __VA_ARGS__);                            \
        } else {                                                                            \
            if ((cache_type) == PWLQ_I8) PWLQ_LANES(KERNEL, f16, int8_t, D, __VA_ARGS__);   \
            else PWLQ_LANES(KERNEL, f16, f16, D, __VA_ARGS__);                              \
        }                                                                                   \
    } while (0)

} // namespace

void append(const pwlq_append_args &g, hipStream_t stream)
{
    Append a = {};
    a.c = cache_of(g.cache);
    a.b = batch_of(g.batch, g.cache);
    a.q = (const char *)g.q.data;
    a.k = (const char *)g.k.data;
    a.v = (const char *)g.v.data;
    a.q_out = (char *)g.q_out.data;
    a.q_stride = g.q.stride, a.q_head = g.q.head_stride;
    a.k_stride = g.k.stride, a.k_head = g.k.head_stride;
    a.v_stride = g.v.stride, a.v_head = g.v.head_stride;
    a.out_stride = g.q_out.stride, a.out_head = g.q_out.head_stride;
    a.q_heads = g.q.data ? g.q_heads : 0;
    a.pairs = g.rotated / 2;
    a.interleaved = g.interleaved;
    a.positions = g.positions;
    a.frequencies = g.frequencies;
    // Few rows: one to a workgroup, its heads shared out among workgroups so that each group of lanes has one (one row of 32 + 16 heads 3.3 us, two
    // to a group 3.7, three 4.4).  Many: two to a workgroup and all heads, so that angles are few and workgroups enough (3795 rows 21.3 us; one row
    // 22.6, four 24.6).
    const int all = a.q_heads + 2 * a.c.heads;
    a.rows = a.b.T >= 1024 ? 2 : 1;
    const int groups = a.c.D <= 16 ? 128 : a.c.D <= 32 ? 64 : a.c.D <= 64 ? 32 : a.c.D <= 128 ? 16 : 8;
    a.heads_each = a.rows > 1 ? all : groups;
    const dim3 grid((unsigned)((a.b.T + a.rows - 1) / a.rows), (unsigned)((all + a.heads_each - 1) / a.heads_each));
    PWLQ_TYPES(k_append, g.k.type, g.cache.type, a.c.D, <<<grid, 256, 0, stream>>>(a));
}

void read(const pwlq_read_args &g, hipStream_t stream)
{
    // few rows one to a workgroup (64 rows 2.9 us, four to one 5.0)
    Read a = {cache_of(g.cache), batch_of(g.batch, g.cache), (char *)g.k.data, (char *)g.v.data,
              g.k.stride, g.k.head_stride, g.v.stride, g.v.head_stride, g.batch.T >= 1024 ? kRows : 1};
    const unsigned grid = (unsigned)((a.b.T + a.rows - 1) / a.rows);
    PWLQ_TYPES(k_read, g.k.data ? g.k.type : g.v.type, g.cache.type, a.c.D, <<<grid, 256, 0, stream>>>(a));
}

} // namespace pwlq_attention
