// Attention over the paged cache: what its kernels share.
//
//   s = scale (q . k), capped by a tanh, less slope |own - slot|;  out = sum softmax(s) v
//
// A query row is one head of one row of the call.  The rows of a sequence whose heads read the same head of the cache are
// taken together, `group` heads of each row of the call after the other, in tiles: a tile's keys and values are read once for
// all of them.  One pass over the keys keeps for each row a reference m, the sum of exp2(s - m) and the sum of exp2(s - m) v;
// s is in units of log 2.
//
// Keys of an item (a tile and a head of the cache) may be split among workgroups.  All items' units of keys lie one after the other
// on a line, which is cut into equal parts, so lengths may differ as they like; lengths are known on the device only.  A part
// that is no whole item leaves its sums in the workspace, and k_attend_join puts them together in the order of the keys.
#pragma once

#include <initializer_list>

#include "launch.h"
#include "cache.h"

namespace pwlq_attention {

struct Stretch;
struct Attend {
    Cache c;
    Batch b;
    const char *q;
    char *out;
    int64_t q_stride, q_head, out_stride, out_head;
    int group;                           // heads of queries for one of the cache
    uint64_t per_group;                  // ceil(2^40 / group)
    float scale, cap;
    const float *slopes;
    int window;                          // 0: none
    const int32_t *prefix;
    const uint64_t *tree;
    int tree_words;
    int tiles;                           // numbers of tiles, of which some may stand for none
    int each;                            // without starts: tiles of a sequence
    int parts;                           // workgroups that the line is cut for; 0: a workgroup for each item
    int least;                           // units of a part, at least,
    int alone;                           // and where that leaves no more parts than CUs: a second workgroup there pays for longer ones
    int *part;                           // workspace: units of a part,
    struct Stretch *stretches;           // of the tiles on the line,
    float2 *top_sum;                     // m (-infinity: none) and the sum of each row of two sums for each part,
    float *sums;                         // and their values
};

constexpr int kMostTiles = 2047;         // of a call that is split
constexpr float kLog2e = 1.4426950408889634f;
// The reference is moved when a score passes it by more than this, so that most tiles move no sums.
constexpr float kSlack = 8.0f;
// Below this a reference is off by 2^-15 at most, half a unit in its last place: the weight of the score that it is of rounds to 1.
constexpr float kFar = 1024.0f;
// The reference for a largest score of `top`.  Weights of binary16 are multiples of 2^-24: many that are less, beside one of 1, would be nothing in the
// product and something in their sum (2^20 of 2^-25: 3 % of the output).  So the largest there is 2^7, with the slack 2^15, and 2^-25 of that is lost.
// Far out, where taking off 7 is a rounding, it is 1.
template <typename T> __device__ inline float reference_of(float top)
{
    if (top == -INFINITY) return 0.0f;
    return __is_same(T, f16) && fabsf(top) < kFar ? top - 7.0f : top;
}

// n / group for 0 <= n < 2^30: what per_group is too large by adds less than n / 2^40 <= 1 / group.  A division takes 25 instructions, and those that
// run once before the first key are fetched once each, which is what they cost.
__device__ inline int by_group(const Attend &a, int n) { return (int)((uint64_t)(uint32_t)n * a.per_group >> 40); }

// A tile: rows first to first + M - 1 of a sequence's `rows` query rows, and the slots that any of them may see.
struct Tile {
    int s, first, rows, prefix, lo, hi;
    Sequence q;
    __device__ bool none() const { return first < 0 || first >= rows; }
};
__device__ inline int tile_key(const Attend &a, int start, int s, int M) { return min(max(start, 0), a.b.T) * a.group / M + s; }

__device__ inline Tile tile_of(const Attend &a, int s, int i, Sequence q, int M)
{
    Tile t;
    t.s = s;
    t.q = q;
    t.first = i * M;
    t.rows = q.rows * a.group;
    t.prefix = a.prefix ? min(max(a.prefix[s], 0), q.length) : 0;
    t.lo = t.hi = 0;
    if (t.none()) return t;
    const int j0 = by_group(a, t.first), j1 = by_group(a, min(t.first + M, t.rows) - 1), kept = q.kept();
    if (a.tree) t.hi = q.length;
    else {
        t.hi = min(max(max(kept + j1 + 1, t.prefix), 0), q.length);
        if (a.window && !t.prefix) t.lo = min(max(kept + j0 - a.window + 1, 0), t.hi);
    }
    return t;
}
// The same for all lanes, and said to be: branches on it are the wavefront's.
__device__ inline Tile uniform(Tile t)
{
    for (int *p : {&t.s, &t.first, &t.rows, &t.prefix, &t.lo, &t.hi, &t.q.start, &t.q.rows, &t.q.length}) *p = __builtin_amdgcn_readfirstlane(*p);
    return t;
}
// Tile number u; s found by one wavefront, or known.
__device__ inline Tile tile(const Attend &a, int u, int M)
{
    int s, i;
    if (a.b.starts) {
        s = find_rising(a.b.S, u, [&](int k) { return tile_key(a, a.b.starts[k], k, M); });
        i = u - tile_key(a, a.b.starts[s], s, M);
    } else {
        s = u / a.each;
        i = u - s * a.each;
    }
    return uniform(tile_of(a, s, i, sequence(a.b, s), M));
}
// Units of keys of a tile: one at least, where its rows get zeros.
__device__ inline int units_of(const Tile &t, int unit) { return t.none() ? 0 : max((t.hi + unit - 1) / unit - t.lo / unit, 1); }

// An item has so many units more on the line, before its first one, for what a workgroup does beside its keys: queries, masks, the first keys' way
// and the sums' take 4 to 8 us, a unit 1.2 to 2.4.  Without it a part of many short items takes twice as long as one of a long one.
constexpr int kSetup = 3;
__device__ inline int length_of(int units) { return units ? units + kSetup : 0; }

// Where a tile lies on the line (of one head), its units, and which rows it has; as it is read by the join.
struct alignas(32) Stretch {
    uint32_t begin, units;
    int first, rows, start;
    __device__ Stretch(uint32_t begin, int units, const Tile &t) : begin(begin), units((uint32_t)units), first(t.first), rows(t.rows), start(t.q.start) {}
};

// Sum over the threads before this one, and over all, in a workgroup of THREADS.  `slots`: LDS of a word for each wavefront, not in use.
template <int THREADS> __device__ inline uint32_t sum_before(uint32_t v, uint32_t *slots, uint32_t &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)s, k);
        if (lane >= k) s += o;
    }
    if (lane == 63) slots[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += slots[w];
        all += slots[w];
    }
    return before + s - v;
}

// Where a workgroup's part of the line begins: places x to end - 1, the first of them place `skip` of head `head` of tile u.
struct Part {
    int x, end, part;                    // the whole line is shorter than 2^31
    int u, head, skip;

    __device__ void cut(const Attend &a, int all)
    {
        const uint32_t line = (uint32_t)all * a.c.heads;
        part = max(max((int)((line + a.parts - 1) / a.parts), min((int)((line + 255) / 256), a.alone)), a.least);
        x = min((uint32_t)blockIdx.x * (uint32_t)part, line);
        end = min((uint32_t)x + (uint32_t)part, line);
        u = head = skip = 0;
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.part = part;
    }
    __device__ void start(const Attend &a, int tile, int begin, int length)
    {
        const uint32_t into = (uint32_t)(x - begin * a.c.heads);
        u = __builtin_amdgcn_readfirstlane(tile);
        head = __builtin_amdgcn_readfirstlane((int)(into / (uint32_t)length));
        skip = __builtin_amdgcn_readfirstlane((int)into) - head * length;
    }
};

// The line of up to 64 tiles of up to 64 sequences, each wavefront for itself: a lane has a tile.  The tiles stay in LDS.  The first workgroup
// leaves the line in the workspace too, for the join.
constexpr int kFewTiles = 64;
template <int M, int UNIT> __device__ Part plan_few(const Attend &a, Tile *tiles)
{
    const int lane = threadIdx.x & 63, u = min(lane, a.tiles - 1);
    int s, i, start, end;
    if (a.b.starts) {
        const int mine = a.b.starts[min(lane, a.b.S - 1)], key = tile_key(a, mine, lane, M);
        int lo = 0, hi = a.b.S;                             // the last s whose tiles begin at u or before
#pragma unroll
        for (int k = 0; k < 6; ++k) {
            const int mid = (lo + hi) / 2;
            const bool below = __shfl(key, mid) <= u;
            if (hi - lo > 1) (below ? lo : hi) = mid;
        }
        s = lo;
        start = a.b.starts[s];
        end = a.b.starts[s + 1];
        i = u - tile_key(a, start, s, M);
    } else {
        s = u / a.each;
        i = u - s * a.each;
        start = s;
        end = s + 1;
    }
    const Tile t = tile_of(a, s, i, sequence(a.b, s, start, end, a.b.lengths[s]), M);
    const int units = lane < a.tiles ? units_of(t, UNIT) : 0;
    const int length = length_of(units);
    uint32_t stop = (uint32_t)length;                       // and so its end on the line
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)stop, k);
        if (lane >= k) stop += o;
    }
    Part p;
    p.cut(a, __builtin_amdgcn_readlane((int)stop, 63));
    if (blockIdx.x == 0 && threadIdx.x < a.tiles) a.stretches[lane] = Stretch(stop - length, units, t);
    if (threadIdx.x < a.tiles) tiles[lane] = t;
    if (p.x < p.end) {
        const int at = __builtin_ctzll(__ballot((int)stop * a.c.heads > p.x));
        const int n = __builtin_amdgcn_readlane(length, at);
        p.start(a, at, __builtin_amdgcn_readlane((int)stop, at) - n, n);
    }
    __syncthreads();
    return p;
}

// The line of more, by the workgroup, in LDS (`room`: kPlanBytes, aligned to a word; free again on return): a word for each wavefront, where each tile
// begins and the line's end, and the starts.
constexpr int kPlanWaves = 8, kPlanBytes = 4 * (kPlanWaves + 2 * (kMostTiles + 1));
template <int M, int UNIT, int THREADS> __device__ Part plan(const Attend &a, uint32_t *room)
{
    static_assert(THREADS <= 64 * kPlanWaves, "LDS");
    uint32_t *const slots = room, *const begin = room + kPlanWaves;
    int32_t *const starts = (int32_t *)(begin + kMostTiles + 1);
    const int each = (a.tiles + THREADS - 1) / THREADS, from = min((int)threadIdx.x * each, a.tiles), to = min(from + each, a.tiles);
    if (a.b.starts) {
        for (int i = threadIdx.x; i <= a.b.S; i += THREADS) starts[i] = a.b.starts[i];
        __syncthreads();
    }
    auto tile_at = [&](int u) {
        if (!a.b.starts) {
            const int s = u / a.each;
            return tile_of(a, s, u - s * a.each, sequence(a.b, s), M);
        }
        int lo = 0, hi = a.b.S;                             // the last s whose tiles begin at u or before
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (tile_key(a, starts[mid], mid, M) <= u) lo = mid;
            else hi = mid;
        }
        return tile_of(a, lo, u - tile_key(a, starts[lo], lo, M), sequence(a.b, lo, starts[lo], starts[lo + 1], a.b.lengths[lo]), M);
    };
    uint32_t mine = 0;
    for (int u = from; u < to; ++u) {
        const int n = length_of(units_of(tile_at(u), UNIT));
        begin[u] = (uint32_t)n;
        mine += (uint32_t)n;
    }
    uint32_t all, at = sum_before<THREADS>(mine, slots, all);
    for (int u = from; u < to; ++u) {
        const uint32_t n = begin[u];
        begin[u] = at;
        if (blockIdx.x == 0) a.stretches[u] = Stretch(at, n ? (int)n - kSetup : 0, tile_at(u));
        at += n;
    }
    if (threadIdx.x == 0) begin[a.tiles] = all;
    __syncthreads();
    Part p;
    p.cut(a, (int)all);
    if (p.x < p.end) {
        int lo = 0, hi = a.tiles;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((int)begin[mid] * a.c.heads <= p.x) lo = mid;
            else hi = mid;
        }
        p.start(a, lo, (int)begin[lo], (int)(begin[lo + 1] - begin[lo]));
    }
    __syncthreads();
    return p;
}

// The segments of a workgroup, one after the other: units begin to stop - 1 of a tile for a head of the cache, counted from
// slot 0, and which of the workspace's sums they leave (-1: a whole item, which needs none).
template <int M, int UNIT, int THREADS> struct Segments {
    Tile t;
    int head, begin, stop, sums;
    Part p;
    int64_t item;
    int units;                           // of t; -1: not looked up

    const Tile *tiles;                   // in LDS, or NULL

    // `few`: LDS for kFewTiles tiles
    __device__ Segments(const Attend &a, uint32_t *room, Tile *few) : item(blockIdx.x), units(-1), tiles(nullptr)
    {
        if (a.parts == 0) return;
        if (a.tiles <= kFewTiles && a.b.S <= kFewTiles) {
            p = plan_few<M, UNIT>(a, few);
            tiles = few;
        } else {
            p = plan<M, UNIT, THREADS>(a, room);
        }
    }
    __device__ bool next(const Attend &a)
    {
        if (a.parts == 0) {
            for (; item < (int64_t)a.tiles * a.c.heads; item += gridDim.x) {
                // the last tiles, which see most, begin first; the workgroups of one head of the cache are on the same L2s
                head = (int)(item % a.c.heads);
                t = tile(a, a.tiles - 1 - (int)(item / a.c.heads), M);
                if (t.none()) continue;
                begin = t.lo / UNIT;
                stop = begin + units_of(t, UNIT);
                sums = -1;
                item += gridDim.x;
                return true;
            }
            return false;
        }
        while (p.x < p.end) {
            while (units <= 0) {
                if (p.u >= a.tiles) return false;
                t = tiles ? uniform(tiles[p.u]) : tile(a, p.u, M);
                units = units_of(t, UNIT);
                if (units == 0) ++p.u;
            }
            const int n = min(units + kSetup - p.skip, p.end - p.x);
            if (n <= 0) return false;                       // starts that do not rise: the line does not fit them
            const int from = max(p.skip - kSetup, 0), to = max(p.skip + n - kSetup, 0);
            head = p.head;
            begin = t.lo / UNIT + from;
            stop = t.lo / UNIT + to;
            // its sums are the first of the part if the item began before the part or with it
            sums = from == 0 && to == units ? -1 : 2 * (int)blockIdx.x + (p.x - p.skip > (int)blockIdx.x * p.part);
            p.x += n;
            p.skip = 0;
            const bool any = to > from;
            if (++p.head == a.c.heads) {
                p.head = 0;
                ++p.u;
                units = -1;
            }
            if (any) return true;
        }
        return false;
    }
};

// --------------------------------------------------------------------------
// a row's scores
// --------------------------------------------------------------------------
// Plain ones as the product has them; sloped: less a bias that grows with the distance; capped, and sloped if there are slopes.
enum Scores { kPlain, kSloped, kCapped };

// cap tanh(y) log2(e) for N values of y = x / cap; cap2 = cap log2(e).  Below a half by a polynomial in y^2, which interpolates tanh(y) / y at
// Chebyshev points and is off by at most 6e-7 of it; above by 1 - 2 / (exp(2y) + 1), which would lose what it subtracts for small y.  Scores are mostly
// well below the cap: a wavefront of which all are takes 5 vector instructions for each.
__device__ inline float cap_near(float y, float cap2)
{
    const float z = y * y;
    return y * __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -0.0443927384f * cap2, 0.131899394f * cap2), -0.333262842f * cap2), 0.999999451f * cap2);
}
typedef float v16f __attribute__((ext_vector_type(16)));
// ... the rest is a function of its own, so that it takes no registers from what is not rare.
__device__ __attribute__((noinline)) v16f cap_far(v16f y, float cap2)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float far = cap2 - 2.0f * cap2 * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(y[i] * (2.0f * kLog2e)) + 1.0f);
        y[i] = fabsf(y[i]) >= 0.5f ? far : cap_near(y[i], cap2);
    }
    return y;
}
template <int N> __device__ inline void cap_scores(float (&y)[N], float cap2)
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(y[i]));
    // a NaN is no maximum: the polynomial keeps it
    if (!__ballot(most >= 0.5f)) {
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = cap_near(y[i], cap2);
    } else {
        v16f x = {};
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = y[i];
        x = cap_far(x, cap2);
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = x[i];
    }
}

// What a lane knows of its query row: it sees slots lo to hi - 1 and those below `prefix`, and where there is a tree those from kept to length - 1
// whose bits are set.
struct RowState {
    int own, lo, hi, prefix;
    float slope;                         // in units of log 2
    uint64_t bits;                       // of the tree's first word
    const uint64_t *words;
};
__device__ inline RowState row_state(const Attend &a, const Tile &t, int row, int head)
{
    RowState r = {-1, 0, 0, 0, 0.0f, 0, nullptr};
    if (row >= t.rows) return r;
    const int j = by_group(a, row), h = head * a.group + row - j * a.group, kept = t.q.kept();
    if (a.slopes) r.slope = a.slopes[h] * kLog2e;
    if (kept + j < 0) return r;
    r.own = kept + j;
    if (a.tree) {
        r.hi = max(kept, 0);
        r.words = a.tree + (int64_t)(t.q.start + j) * a.tree_words;
        r.bits = r.words[0];
    } else {
        r.hi = min(r.own + 1, t.q.length);
        if (a.window) r.lo = max(r.own - a.window + 1, 0);
        r.prefix = t.prefix;
    }
    return r;
}
// Bits 0 to n - 1, n any number.
__device__ inline uint64_t low_bits(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }
// Which of the 64 slots from `from` on the row sees, as bits.
__device__ inline uint64_t seen_slots(const Attend &a, const Tile &t, const RowState &r, int from)
{
    uint64_t seen = (low_bits(r.hi - from) & ~low_bits(r.lo - from)) | low_bits(r.prefix - from);
    if (a.tree) {
        const int j = from - t.q.kept();                    // the first slot's row in the tree
        if (a.tree_words == 1) {
            if (r.own >= 0 && j > -64 && j < 64) seen |= j >= 0 ? r.bits >> j : r.bits << -j;
        } else if (r.own >= 0 && j > -64) {
            const int word = j >> 6, shift = j & 63;       // of the first slot, from -1 on
            const uint64_t low = word >= 0 && word < a.tree_words ? r.words[word] : 0;
            const uint64_t high = word + 1 < a.tree_words ? r.words[word + 1] : 0;
            seen |= shift ? low >> shift | high << (64 - shift) : low;
        }
        seen &= low_bits(t.q.length - from);
    }
    return seen;
}
// The slots that rows first to last (of the tile's sequence) all see: begin to end - 1, and those below prefix.
struct Common {
    int prefix, begin, end;
    __device__ bool has(int from, int stop) const { return stop <= prefix || (from >= begin && stop <= end); }
};
__device__ inline Common common(const Attend &a, const Tile &t, int first, int last)
{
    const int kept = t.q.kept(), j0 = by_group(a, first), j1 = by_group(a, last);
    Common c = {0, 0, 0};
    if (kept + j0 < 0) return c;
    c.prefix = t.prefix;
    c.end = a.tree ? kept : min(kept + j0 + 1, t.q.length);
    if (a.window) c.begin = kept + j1 - a.window + 1;
    return c;
}

// --------------------------------------------------------------------------
// matrix instructions, and vectors of 16-bit elements
// --------------------------------------------------------------------------
typedef short v4s __attribute__((ext_vector_type(4)));

__device__ inline v4f mfma16(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline v4f mfma16(v8h a, v8h b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline v16f mfma32(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline v16f mfma32(v8h a, v8h b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

template <typename T> __device__ inline typename Vec8<T>::type as8(v4u w)
{
    union { v4u w; typename Vec8<T>::type v; } u;
    u.w = w;
    return u.v;
}
template <typename T> __device__ inline v4u words(typename Vec8<T>::type v)
{
    union { typename Vec8<T>::type v; v4u w; } u;
    u.v = v;
    return u.w;
}
// Eight codes as T, times a factor.
template <typename T> __device__ inline typename Vec8<T>::type codes8(uint32_t a, uint32_t b)
{
    return __builtin_convertvector(pwlq_block::widen(v2u{a, b}), typename Vec8<T>::type);
}
template <typename T> __device__ inline typename Vec8<T>::type codes8(uint32_t a, uint32_t b, float factor)
{
    v8f w = pwlq_block::widen(v2u{a, b});
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] *= factor;
    return __builtin_convertvector(w, typename Vec8<T>::type);
}

// Sixteen bytes of the cache; rows are whole numbers of them, at their alignment.
__device__ inline v4u load16(const char *p) { return *(const v4u *)p; }

// Four neighbouring rows' elements of one column, for each of sixteen columns: a group of sixteen lanes reads four rows of sixteen
// elements from LDS, lane l the four of row l / 4 from column 4 (l % 4) on, and gets column l.
__device__ inline v4s read_columns(const char *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p);
}
template <typename T> __device__ inline typename Vec8<T>::type columns8(const char *p, const char *q)
{
    union { v4s h[2]; typename Vec8<T>::type v; } u;
    u.h[0] = read_columns(p);
    u.h[1] = read_columns(q);
    return u.v;
}

// Infinities and NaN among 16-bit elements: bit 15 of each half where its exponent is all ones.
template <typename T> __device__ inline uint32_t not_finite(uint32_t w)
{
    constexpr uint32_t exponent = sizeof(T) == 2 && __is_same(T, bf16) ? 0x7f807f80u : 0x7c007c00u;
    constexpr uint32_t one = __is_same(T, bf16) ? 0x00800080u : 0x04000400u;
    return ((w & exponent) + one) & 0x80008000u;
}
// ... taken out; whether there were any.
template <typename T> __device__ inline bool make_finite(v4u &v)
{
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t bad = not_finite<T>(v[i]);
        any |= bad;
        v[i] &= ~((bad >> 15) * 0xffffu);
    }
    return any != 0;
}
// Where some rows do not see all keys, a value that is not finite must reach the rows that see it and no others, and 0 times it would be NaN.  So
// such values are taken out of the product.  An item's end, where its sums are all that is left in registers, adds what they are for the
// rows that see them: two more products, with 1 for each key that a row sees, count them and add their signs; as many as the sum says are
// infinities of one sign.  The values are read again, one by one, in the operand's layout: channel d of slots `from` to from + 3 and from + apart to
// from + apart + 3.  `seen`: bits 0 to 3 and 4 to 7, of those slots.
template <typename T, typename C> struct NotFinite {
    typename Vec8<T>::type counts, signs, ones;

    __device__ NotFinite(const Attend &a, const int32_t *table, int head, int from, int apart, int end, int d, uint32_t seen)
    {
        uint32_t bad = 0, plus = 0, minus = 0;
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            const int slot = from + (i & 3) + (i / 4) * apart;
            if (slot >= end || d >= a.c.D) continue;
            const int page = table[slot >> a.c.shift];
            if ((unsigned)page >= (unsigned)a.c.pages) continue;
            const int64_t row = row_number(a.c, Place{page, slot & ((1 << a.c.shift) - 1)}, head);
            float v = pwlq_block::widen(((const C *)a.c.values)[row * a.c.D + d]);
            if constexpr (sizeof(C) == 1) v = (float)(T)(v * a.c.value_step[row]);
            bad |= (uint32_t)!(fabsf(v) < INFINITY) << i;
            plus |= (uint32_t)(v == INFINITY) << i;
            minus |= (uint32_t)(v == -INFINITY) << i;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            counts[i] = bad >> i & 1 ? (T)1.0f : (T)0.0f;
            signs[i] = plus >> i & 1 ? (T)1.0f : minus >> i & 1 ? (T)-1.0f : (T)0.0f;
            ones[i] = seen >> i & 1 ? (T)1.0f : (T)0.0f;
        }
    }
};
__device__ inline float not_finite_sum(float count, float sign)
{
    return count == 0.0f ? 0.0f : count == fabsf(sign) ? copysignf(INFINITY, sign) : __builtin_nanf("");
}

typedef float loose4f __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> __device__ inline void store4(char *p, v4f v)
{
    typedef T v4 __attribute__((ext_vector_type(4)));
    typedef T loose __attribute__((ext_vector_type(4), aligned(2)));
    *(loose *)p = __builtin_convertvector(v, v4);
}

} // namespace pwlq_attention
