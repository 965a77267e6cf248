// k_attend_few: tiles of 16 or 32 query rows, for single tokens and small trees.
//
// Bound by memory: keys and values are read once, with matrix instructions as good as idle (16 rows against 32 keys of 128
// channels take 256 of their cycles for 16 KiB).  Each of the four wavefronts takes 32 keys of a unit of 128 by itself, with
// no barrier until an item's end.  8 heads of 128 channels, join included: a token of 64 sequences of up to 8192 rows 201 us (1.1 GB, 5.5 TB/s), of one of
// 131072 rows in 8 bits 61 (4.5 TB/s), of one of 1001 rows 11, which is latencies; 16 heads of 256 channels and a window of 1024 in 16 sequences 38 (3.3
// TB/s: 256 registers of a lane for sums and keys leave room for one workgroup on a CU).
//
// S^T = K Q^T: a lane holds one query row's scores of four neighbouring keys, and as the product's reduction index may be in any
// order, they are the operand of O^T = V^T P^T as they are.  Keys come from memory in the operand's layout; values pass through
// LDS, whose transposing read gives a lane one channel of four keys.
#pragma once

#include "attend.h"

namespace pwlq_attention {

template <typename T, typename C, int DP, int RB> struct Few {
    static constexpr bool kCodes = sizeof(C) == 1, kMayBeBad = !kCodes || __is_same(T, f16);     // values that are not finite
    static constexpr int kUnit = 128, kRows = 16 * RB;
    static constexpr int kSteps = DP / 32, kColumns = DP / 16;
    static constexpr int kLoads = kCodes ? DP / 64 : DP / 32;                      // of 16 bytes, for 16 keys
    static constexpr int kChunks = kCodes ? DP / 16 : DP / 8;                      // of 16 bytes, of a row of values
    static constexpr int kValueRows = 64 / kChunks, kValueLoads = 32 / kValueRows;
    static constexpr int kStride = 2 * DP + 64;                                    // bytes of a row of values in LDS: four rows, all banks
    static constexpr int kSumStride = DP + 4;                                      // floats of a row of sums in LDS
    static constexpr int kRoom = 4 * 32 * kStride;
    static_assert(kRoom >= 4 * 16 * kSumStride * 4 && kRoom >= kPlanBytes, "LDS");
    typedef typename Vec8<T>::type v8;

    v4u k[2][kLoads], v[kValueLoads];
    v4f key_step[2], value_step[2];
    float row_step[kValueLoads];                                                   // of values' rows, where they are scaled as they are read

    // 32 keys: blocks of sixteen from slot `from` on, on pages p[0] and p[1]
    __device__ void load(const Attend &a, int head, int from, const int *p, int lane)
    {
        const int D = a.c.D, row = lane & 15, quarter = lane >> 4;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t n = row_number(a.c, Place{max(p[b], 0), (from + 16 * b) & ((1 << a.c.shift) - 1)}, head);
            const char *const keys = a.c.keys + n * D * (int)sizeof(C), *const values = a.c.values + n * D * (int)sizeof(C);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int d = kCodes ? 64 * j + 16 * quarter : 32 * j + 8 * quarter;
                k[b][j] = load16(keys + (uint32_t)((row * D + (d < D ? d : 0)) * (int)sizeof(C)));
            }
#pragma unroll
            for (int j = b * kValueLoads / 2; j < (b + 1) * kValueLoads / 2; ++j) {
                const int r = (j * kValueRows) % 16 + lane / kChunks, d = lane % kChunks * (16 / (int)sizeof(C));
                v[j] = load16(values + (uint32_t)((r * D + (d < D ? d : 0)) * (int)sizeof(C)));
                if constexpr (kCodes && __is_same(T, f16)) row_step[j] = a.c.value_step[n + r];
            }
            if constexpr (kCodes) {
                key_step[b] = *(const v4f *)(a.c.key_step + n + 4 * quarter);
                if constexpr (!__is_same(T, f16)) value_step[b] = *(const v4f *)(a.c.value_step + n + 4 * quarter);
            }
        }
    }

    // Values to LDS.  `checked`: some row does not see all keys; then what is past the end is 0, and infinities and NaN before it are taken
    // out and reported.
    __device__ bool put_values(const Attend &a, char *room, int lane, bool checked, int from, int end, const int *p) const
    {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < kValueLoads; ++j) {
            const int r = j * kValueRows + lane / kChunks, chunk = lane % kChunks;
            char *const to = room + r * kStride;
            if constexpr (kCodes) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    v8 w;
                    if constexpr (__is_same(T, f16)) {
                        float step = row_step[j];
                        if (checked && (from + r >= end || p[r / 16] < 0)) step = 0.0f;
                        w = codes8<T>(v[j][2 * h], v[j][2 * h + 1], step);
                        if (checked) {
                            v4u u = words<T>(w);
                            bad |= make_finite<T>(u) && chunk * 16 < a.c.D;
                            w = as8<T>(u);
                        }
                    } else {
                        w = codes8<T>(v[j][2 * h], v[j][2 * h + 1]);
                    }
                    *(v4u *)(to + 32 * chunk + 16 * h) = words<T>(w);
                }
            } else {
                v4u w = v[j];
                if (checked) {
                    if (from + r >= end || p[r / 16] < 0) w = v4u{0u, 0u, 0u, 0u};
                    bad |= make_finite<T>(w) && chunk * 8 < a.c.D;
                }
                *(v4u *)(to + 16 * chunk) = w;
            }
        }
        return __ballot(bad) != 0;
    }

    __device__ v8 key(const Attend &a, int b, int step, int quarter) const
    {
        if constexpr (kCodes) {
            const v4u w = k[b][step / 2];
            return codes8<T>(w[2 * (step & 1)], w[2 * (step & 1) + 1]);
        } else {
            v4u w = k[b][step];
            if (a.c.D != DP && 32 * step + 8 * quarter >= a.c.D) w = v4u{0u, 0u, 0u, 0u};
            return as8<T>(w);
        }
    }
    // the first of the eight channels that a lane has of step `step`
    static __device__ int channel(int step, int quarter) { return kCodes ? 64 * (step / 2) + 16 * quarter + 8 * (step & 1) : 32 * step + 8 * quarter; }
};

template <typename T, typename C, int DP, int RB, Scores SCORES>
__global__ __launch_bounds__(256, DP * RB > 128 ? 1 : 2) void k_attend_few(const Attend a)
{
    typedef Few<T, C, DP, RB> F;
    typedef typename F::v8 v8;
    __shared__ __attribute__((aligned(16))) char room[F::kRoom];
    __shared__ float2 top_sum[4][F::kRows];
    __shared__ Tile tiles[kFewTiles];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4;
    char *const values = room + wave * 32 * F::kStride;
    const char *const columns = values + (4 * quarter + (lane & 15) / 4) * F::kStride + (lane & 3) * 8;
    const float to_cap = SCORES == kCapped ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;

    Segments<F::kRows, F::kUnit, 256> segments(a, (uint32_t *)room, tiles);
    while (segments.next(a)) {
        const Tile t = segments.t;
        const int head = segments.head, begin = segments.begin, stop = segments.stop, sums = segments.sums;
        // this wavefront's units: 32 keys from 128 u + 32 wave on
        const int first = max(begin, (t.lo - 32 * wave + 96) >> 7), end = min(stop, (t.hi - 32 * wave + 127) >> 7);
        const int32_t *const table = a.b.table + t.s * a.b.table_stride;
        bool bad = false;                                  // a value taken out
        F f;
        int pages = -1, p[2];                              // lane 2i + b: the page of block b of unit base + i
        int base = 0;
        auto find_pages = [&](int u) {
            if (u == first || u - base == 32) {
                base = u;
                const int slot = 128 * (u + lane / 2) + 32 * wave + 16 * (lane & 1);
                pages = -1;
                if (slot < t.hi) {
                    pages = table[slot >> a.c.shift];
                    if ((unsigned)pages >= (unsigned)a.c.pages) pages = -1;
                }
            }
            p[0] = __builtin_amdgcn_readlane(pages, 2 * (u - base));
            p[1] = __builtin_amdgcn_readlane(pages, 2 * (u - base) + 1);
        };
        if (first < end) {
            find_pages(first);
            f.load(a, head, 128 * first + 32 * wave, p, lane);
        }
        // the queries while the first keys are on their way
        v8 q[RB][F::kSteps];
        RowState state[RB];
        v4f acc[RB][F::kColumns];
        float top[RB], reference[RB], sum[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int row = t.first + 16 * r + (lane & 15);
            state[r] = row_state(a, t, row, head);
            const int j = by_group(a, min(row, t.rows - 1)), h = head * a.group + min(row, t.rows - 1) - j * a.group;
            const T *const in = (const T *)a.q + (int64_t)(t.q.start + j) * a.q_stride + h * a.q_head;
#pragma unroll
            for (int s = 0; s < F::kSteps; ++s) {
                const int d = F::channel(s, quarter);
                q[r][s] = v8{};
                if (row < t.rows && d < a.c.D) q[r][s] = pwlq_block::load8<T>(in + d);
            }
#pragma unroll
            for (int c = 0; c < F::kColumns; ++c) acc[r][c] = v4f{};
            top[r] = -INFINITY;
            reference[r] = sum[r] = 0.0f;
        }
        const Common whole = common(a, t, t.first, min(t.first + F::kRows, t.rows) - 1);
        for (int u = first; u < end; ++u) {
            const int from = 128 * u + 32 * wave, now[2] = {p[0], p[1]};
            const bool full = now[0] >= 0 && now[1] >= 0 && whole.has(from, from + 32);
            bad |= f.put_values(a, values, lane, !full, from, t.hi, now);
            v4f s[RB][2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int r = 0; r < RB; ++r) s[r][b] = v4f{};
#pragma unroll
                for (int step = 0; step < F::kSteps; ++step) {
                    const v8 k = f.key(a, b, step, quarter);
#pragma unroll
                    for (int r = 0; r < RB; ++r) s[r][b] = mfma16(k, q[r][step], s[r][b]);
                }
                if constexpr (F::kCodes) {
                    const v4f step = f.key_step[b] * to_cap;
#pragma unroll
                    for (int r = 0; r < RB; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[r][b][i] *= step[i];
                }
            }
            const v4f value_step[2] = {f.value_step[0], f.value_step[1]};
            if (u + 1 < end) {
                find_pages(u + 1);
                f.load(a, head, from + 128, p, lane);
            }
            const uint32_t there = (now[0] < 0 ? 0u : 0xffffu) | (now[1] < 0 ? 0u : 0xffff0000u);
            v8 weight[RB];
#pragma unroll
            for (int r = 0; r < RB; ++r) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = F::kCodes ? s[r][i / 4][i & 3] : s[r][i / 4][i & 3] * to_cap;
                if constexpr (SCORES == kCapped) cap_scores(x, cap2);
                if (SCORES != kPlain && a.slopes) {
                    const float away = (float)(state[r].own - from - 4 * quarter);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = __builtin_fmaf(-state[r].slope, fabsf(away - (float)(16 * (i / 4) + (i & 3))), x[i]);
                }
                if (!full) {
                    const uint32_t mine = ((uint32_t)seen_slots(a, t, state[r], from) & there) >> (4 * quarter);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = mine >> (16 * (i / 4) + (i & 3)) & 1 ? x[i] : -INFINITY;
                }
                float most = x[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) most = fmaxf(most, x[i]);
                if (__ballot(most > top[r] + kSlack)) {
                    most = fmaxf(most, __shfl_xor(most, 16));
                    most = fmaxf(top[r], fmaxf(most, __shfl_xor(most, 32)));
                    const float next = reference_of<T>(most);
                    const float old = top[r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(reference[r] - next);
                    // a sum that is NaN already stays NaN
                    sum[r] *= top[r] == -INFINITY ? 1.0f : old;
#pragma unroll
                    for (int c = 0; c < F::kColumns; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[r][c][i] *= top[r] == -INFINITY ? 1.0f : old;
                    top[r] = most;
                    reference[r] = next;
                }
                // a unit's weights are summed by themselves: one by one they might be nothing beside what there is
                float w[8], more = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = __builtin_amdgcn_exp2f(x[i] - reference[r]);
                    more += w[i];
                }
                sum[r] += more;
                if constexpr (F::kCodes && !__is_same(T, f16)) {
                    // a row's step joins its weight: one rounding to bfloat16, of their product; a step may be NaN
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] *= value_step[i / 4][i & 3];
                    if (!full) {
                        const uint32_t mine = ((uint32_t)seen_slots(a, t, state[r], from) & there) >> (4 * quarter);
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = mine >> (16 * (i / 4) + (i & 3)) & 1 ? w[i] : 0.0f;
                    }
                }
                v8f all;
#pragma unroll
                for (int i = 0; i < 8; ++i) all[i] = w[i];
                weight[r] = __builtin_convertvector(all, v8);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int c = 0; c < F::kColumns; ++c) {
                const v8 v = columns8<T>(columns + 32 * c, columns + 16 * F::kStride + 32 * c);
#pragma unroll
                for (int r = 0; r < RB; ++r) acc[r][c] = mfma16(v, weight[r], acc[r][c]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }

        // the four wavefronts' sums, each with its reference from here on
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            if (top[r] != -INFINITY) top[r] = reference[r];
            sum[r] += __shfl_xor(sum[r], 16);
            sum[r] += __shfl_xor(sum[r], 32);
            if (lane < 16) top_sum[wave][16 * r + lane] = make_float2(top[r], sum[r]);
        }
        __syncthreads();
        float *const all = (float *)room;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            float most = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) most = fmaxf(most, top_sum[w][16 * r + (lane & 15)].x);
            const float factor = top[r] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[r] - most);
#pragma unroll
            for (int c = 0; c < F::kColumns; ++c)
                *(v4f *)(all + (wave * 16 + (lane & 15)) * F::kSumStride + 16 * c + 4 * quarter) = acc[r][c] * factor;
            if (F::kMayBeBad && bad) {
#pragma unroll 1
                for (int c = 0; c < F::kColumns; ++c) {
                    v4f count = {}, sign = {};
                    for (int u = first; u < end; ++u) {
                        const int from = 128 * u + 32 * wave;
                        const uint32_t mine = (uint32_t)(seen_slots(a, t, state[r], from) >> (4 * quarter));
                        const NotFinite<T, C> v(a, table, head, from + 4 * quarter, 16, t.hi, 16 * c + (lane & 15), (mine & 15) | (mine >> 12 & 0xf0));
                        count = mfma16(v.counts, v.ones, count);
                        sign = mfma16(v.signs, v.ones, sign);
                    }
                    v4f *const at = (v4f *)(all + (wave * 16 + (lane & 15)) * F::kSumStride + 16 * c + 4 * quarter);
                    v4f v = *at;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += not_finite_sum(count[i], sign[i]);
                    *at = v;
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < 16 * DP / 4; i += 256) {
                const int of = i / (DP / 4), d = i % (DP / 4) * 4, row = t.first + 16 * r + of;
                if (row >= t.rows || d >= a.c.D) continue;
                v4f v = {};
                float m = -INFINITY, total = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w) m = fmaxf(m, top_sum[w][16 * r + of].x);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float2 o = top_sum[w][16 * r + of];
                    total += o.y * (o.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(o.x - m));
                    v += *(const v4f *)(all + (w * 16 + of) * F::kSumStride + d);
                }
                if (sums >= 0) {
                    const int64_t at = (int64_t)sums * F::kRows + 16 * r + of;
                    *(v4f *)(a.sums + at * DP + d) = v;
                    if (d == 0) a.top_sum[at] = make_float2(m, total);
                } else {
                    const int j = by_group(a, row), h = head * a.group + row - j * a.group;
                    store4<T>(a.out + ((t.q.start + j) * a.out_stride + h * a.out_head + d) * 2, total == 0.0f ? v4f{} : v * (1.0f / total));
                }
            }
            __syncthreads();
        }
    }
}

} // namespace pwlq_attention
