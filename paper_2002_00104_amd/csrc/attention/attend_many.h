// k_attend_many: tiles of 128 query rows, for prompts and larger trees.
//
// Bound by the matrix cores and by the exponentials beside them: a tile of 64 keys takes a wavefront's 32 rows 1024 cycles of matrix
// instructions (128 channels) and as many of vector instructions for its 2048 weights.  Two workgroups share a CU, so one's
// products run beside the other's exponentials.
//
// Keys and values of a tile are staged in LDS, twice: one is filled while the other is worked on, a barrier a tile.  As for few
// rows, S^T = K Q^T leaves a lane its query row's weights in the layout of the operand of O^T = V^T P^T.
#pragma once

#include "attend.h"

namespace pwlq_attention {

template <typename T, typename C, int DP> struct Many {
    static constexpr bool kCodes = sizeof(C) == 1, kScaled = kCodes && __is_same(T, f16);    // values scaled as they are read
    static constexpr int kRows = 128, kKeys = DP == 256 ? 32 : 64;
    static constexpr int kSteps = DP / 16, kColumns = DP / 32, kBlocks = kKeys / 32;
    static constexpr int kChunks = kCodes ? DP / 16 : DP / 8;                      // of 16 bytes, of a row
    static constexpr int kPass = 256 / kChunks, kLoads = kKeys / kPass, kWavePass = 64 / kChunks;
    static constexpr int kKeyStride = 2 * DP + 16, kValueStride = 2 * DP + 64;     // bytes of a row in LDS
    static constexpr int kStage = kKeys * (kKeyStride + kValueStride);
    static_assert(2 * kStage >= 4 * (2 * kMostTiles + 16), "LDS");
    typedef typename Vec8<T>::type v8;

    v4u k[kLoads], v[kLoads];
    float key_step[kLoads], value_step[kLoads];

    // `pages`: lane i has the page of block base + i of sixteen keys
    __device__ void load(const Attend &a, int head, int from, int pages, int base, int wave, int lane)
    {
        const int D = a.c.D, row = lane / kChunks, d = lane % kChunks * (16 / (int)sizeof(C));
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = j * kPass + wave * kWavePass, slot = from + r;
            const int page = __builtin_amdgcn_readlane(pages, (slot >> 4) - base);
            const int64_t n = row_number(a.c, Place{max(page, 0), slot & ((1 << a.c.shift) - 1)}, head);
            const uint32_t offset = (uint32_t)((row * D + (d < D ? d : 0)) * (int)sizeof(C));
            k[j] = load16(a.c.keys + n * D * (int)sizeof(C) + offset);
            v[j] = load16(a.c.values + n * D * (int)sizeof(C) + offset);
            if constexpr (kCodes) {
                key_step[j] = a.c.key_step[n + row];
                value_step[j] = a.c.value_step[n + row];
            }
        }
    }
    // To LDS.  `checked`: some row does not see all keys, see Few::put_values.
    __device__ bool put(const Attend &a, char *room, float *steps, int lane, int wave, bool checked, int from, int end, int pages, int base) const
    {
        char *const keys = room, *const values = room + kKeys * kKeyStride;
        const int chunk = lane % kChunks;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int r = j * kPass + wave * kWavePass + lane / kChunks;
            bool none = false;
            if (checked) none = from + r >= end || __builtin_amdgcn_readlane(pages, ((from + j * kPass + wave * kWavePass) >> 4) - base) < 0;
            if constexpr (kCodes) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    *(v4u *)(keys + r * kKeyStride + 32 * chunk + 16 * h) = words<T>(codes8<T>(k[j][2 * h], k[j][2 * h + 1]));
                    v4u w;
                    if constexpr (kScaled) {
                        w = words<T>(codes8<T>(v[j][2 * h], v[j][2 * h + 1], none ? 0.0f : value_step[j]));
                        if (checked) bad |= make_finite<T>(w) && chunk * 16 < a.c.D;
                    } else {
                        w = words<T>(codes8<T>(v[j][2 * h], v[j][2 * h + 1]));
                    }
                    *(v4u *)(values + r * kValueStride + 32 * chunk + 16 * h) = w;
                }
                if (chunk == 0) {
                    steps[r] = key_step[j];
                    steps[kKeys + r] = value_step[j];
                }
            } else {
                v4u w = k[j], x = v[j];
                if (a.c.D != DP && chunk * 8 >= a.c.D) w = v4u{0u, 0u, 0u, 0u};
                if (checked) {
                    if (none) x = v4u{0u, 0u, 0u, 0u};
                    bad |= make_finite<T>(x) && chunk * 8 < a.c.D;
                }
                *(v4u *)(keys + r * kKeyStride + 16 * chunk) = w;
                *(v4u *)(values + r * kValueStride + 16 * chunk) = x;
            }
        }
        return __ballot(bad) != 0;
    }
};

template <typename T, typename C, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attend_many(const Attend a)
{
    typedef Many<T, C, DP> F;
    typedef typename F::v8 v8;
    __shared__ __attribute__((aligned(16))) char room[2 * F::kStage];
    __shared__ float steps[2][F::kCodes ? 2 * F::kKeys : 4];
    __shared__ int bad_tile[2][4];                         // by wavefront
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const float to_cap = a.cap > 0.0f ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;

    Segments<F::kRows, F::kKeys> segments(a, (uint32_t *)room);
    while (segments.next(a)) {
        const Tile t = segments.t;
        const int head = segments.head, sums = segments.sums;
        const int row = t.first + 32 * wave + (lane & 31), clamped = min(row, t.rows - 1);
        const RowState state = row_state(a, t, row, head);
        const int j = clamped / a.group, h = head * a.group + clamped - j * a.group;
        const T *const in = (const T *)a.q + (int64_t)(t.q.start + j) * a.q_stride + h * a.q_head;
        v8 q[F::kSteps];
#pragma unroll
        for (int s = 0; s < F::kSteps; ++s) {
            const int d = 16 * s + 8 * half;
            q[s] = v8{};
            if (row < t.rows && d < a.c.D) q[s] = pwlq_block::load8<T>(in + d);
        }
        v16f acc[F::kColumns];
#pragma unroll
        for (int c = 0; c < F::kColumns; ++c) acc[c] = v16f{};
        float top = -INFINITY, reference = 0.0f, sum = 0.0f;

        const int last = min(t.first + F::kRows, t.rows) - 1;
        // this wavefront's rows, and the slots that any of them may see
        const int my_first = min(t.first + 32 * wave, last), my_last = min(my_first + 31, last);
        const bool mine = t.first + 32 * wave <= last;
        int my_end = t.hi, my_begin = t.lo;
        if (!a.tree) {
            my_end = min(max(t.q.kept() + my_last / a.group + 1, t.prefix), t.hi);
            if (a.window && !t.prefix) my_begin = max(t.q.kept() + my_first / a.group - a.window + 1, t.lo);
        }
        const int32_t *const table = a.b.table + t.s * a.b.table_stride;
        const int begin = segments.begin, end = min(segments.stop, (t.hi + F::kKeys - 1) / F::kKeys);
        F f;
        int pages = -1, base = 0;
        auto find_pages = [&](int from, bool first) {      // of the blocks of the tile at `from`
            if (first || (from >> 4) - base == 64) {
                base = from >> 4;
                const int slot = 16 * (base + lane);
                pages = -1;
                if (slot < t.hi) {
                    pages = table[slot >> a.c.shift];
                    if ((unsigned)pages >= (unsigned)a.c.pages) pages = -1;
                }
            }
        };
        // whether all rows of the tile see all keys from `from` on
        auto whole = [&](int from) {
            bool there = true;
#pragma unroll
            for (int b = 0; b < F::kKeys / 16; ++b) there = there && __builtin_amdgcn_readlane(pages, (from >> 4) - base + b) >= 0;
            return there && all_see(a, t, t.first, last, from, from + F::kKeys);
        };
        bool full = false;
        uint32_t lacks = 0;                                // blocks without a page of the tile that is worked on
        auto put = [&](int from, int to) {
            full = whole(from);
            lacks = 0;
#pragma unroll
            for (int b = 0; b < F::kKeys / 16; ++b) lacks |= (uint32_t)(__builtin_amdgcn_readlane(pages, (from >> 4) - base + b) < 0) << b;
            const bool bad = f.put(a, room + to * F::kStage, steps[to], lane, wave, !full, from, t.hi, pages, base);
            if (lane == 0) bad_tile[to][wave] = bad;
        };
        if (begin < end) {
            find_pages(begin * F::kKeys, true);
            f.load(a, head, begin * F::kKeys, pages, base, wave, lane);
            put(begin * F::kKeys, 0);
        }
        __syncthreads();
        for (int u = begin; u < end; ++u) {
            const int at = (u - begin) & 1, from = u * F::kKeys;
            const bool all_full = full;
            const uint32_t none = lacks;
            if (u + 1 < end) {
                find_pages(from + F::kKeys, false);
                f.load(a, head, from + F::kKeys, pages, base, wave, lane);
            }
            if (mine && from < my_end && from + F::kKeys > my_begin) {
                const char *const keys = room + at * F::kStage + (lane & 31) * F::kKeyStride + 16 * half;
                const char *const values = room + at * F::kStage + F::kKeys * F::kKeyStride +
                                           (4 * half + (lane & 15) / 4) * F::kValueStride + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
                const bool my_full = all_full || (!none && all_see(a, t, my_first, my_last, from, from + F::kKeys));
                v16f s[F::kBlocks];
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b) {
                    s[b] = v16f{};
#pragma unroll
                    for (int step = 0; step < F::kSteps; ++step)
                        s[b] = mfma32(as8<T>(*(const v4u *)(keys + b * 32 * F::kKeyStride + 32 * step)), q[step], s[b]);
                }
                // element i of block b is key 32 b + 8 (i / 4) + 4 half + i % 4
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b) {
                    if constexpr (F::kCodes) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const v4f step = *(const v4f *)(steps[at] + 32 * b + 2 * i + 4 * half);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[b][i + e] *= step[e];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] *= to_cap;
                    if (a.cap > 0.0f) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[b][i] = capped(s[b][i], cap2);
                    }
                    if (a.slopes) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            s[b][i] -= state.slope * (float)abs(state.own - (from + 32 * b + 8 * (i / 4) + 4 * half + (i & 3)));
                    }
                }
                uint32_t see[F::kBlocks];
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b) see[b] = 0xffff;
                if (!my_full) {
#pragma unroll
                    for (int b = 0; b < F::kBlocks; ++b) {
                        see[b] = 0;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int key = 32 * b + 8 * (i / 4) + 4 * half + (i & 3);
                            const bool seen_it = !(none >> (2 * b + i / 8) & 1) & sees(a, t, state, from + key);
                            see[b] |= (uint32_t)seen_it << i;
                            s[b][i] = seen_it ? s[b][i] : -INFINITY;
                        }
                    }
                }
                float most = -INFINITY;
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, s[b][i]);
                if (__ballot(most > top + kSlack)) {
                    most = fmaxf(top, fmaxf(most, __shfl_xor(most, 32)));
                    const float next = most == -INFINITY ? 0.0f : most;
                    // a sum that is NaN already stays NaN
                    const float old = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(reference - next);
                    sum *= old;
#pragma unroll
                    for (int c = 0; c < F::kColumns; ++c)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[c][i] *= old;
                    top = most;
                    reference = next;
                }
                uint32_t above[F::kBlocks];
                v8 weight[F::kBlocks][2];
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[b][i] = __builtin_amdgcn_exp2f(s[b][i] - reference);
                        if (!my_full && !(see[b] >> i & 1)) s[b][i] = 0.0f;
                        sum += s[b][i];
                    }
                    above[b] = 0;
                    if (!all_full) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) above[b] |= (s[b][i] > 0.0f ? 1u : 0u) << i;
                    }
                    if constexpr (F::kCodes && !F::kScaled) {
                        // a row's step joins its weight: one rounding to bfloat16, of their product
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const v4f step = *(const v4f *)(steps[at] + F::kKeys + 32 * b + 2 * i + 4 * half);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                s[b][i + e] = !my_full && !(see[b] >> (i + e) & 1) ? 0.0f : s[b][i + e] * step[e];
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        v8f w;
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = s[b][8 * e + i];
                        weight[b][e] = __builtin_convertvector(w, v8);
                    }
                }
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int c = 0; c < F::kColumns; ++c) {
                            const char *const p = values + (32 * b + 16 * e) * F::kValueStride + 64 * c;
                            acc[c] = mfma32(columns8<T>(p, p + 8 * F::kValueStride), weight[b][e], acc[c]);
                        }
                if (!all_full && (bad_tile[at][0] | bad_tile[at][1] | bad_tile[at][2] | bad_tile[at][3])) {
                    // infinities and NaN among the values, of which some rows see less than all: row by row and key by key
                    uint32_t other_see[F::kBlocks], other_above[F::kBlocks];
#pragma unroll
                    for (int b = 0; b < F::kBlocks; ++b) {
                        other_see[b] = __shfl_xor(see[b], 32);
                        other_above[b] = __shfl_xor(above[b], 32);
                    }
                    for (int key = 0; key < F::kKeys && from + key < t.hi; ++key) {
                        if (none >> (key / 16) & 1) continue;
                        const int64_t n = row_number(a.c, Place{table[(from + key) >> a.c.shift], (from + key) & ((1 << a.c.shift) - 1)}, head);
                        const int bit = (key & 3) + 4 * ((key >> 3) & 3);
                        const bool own = ((key >> 2) & 1) == half;
                        uint32_t sees_it = 0, weighs = 0;
#pragma unroll
                        for (int b = 0; b < F::kBlocks; ++b)
                            if (b == key / 32) {
                                sees_it = (own ? see[b] : other_see[b]) >> bit & 1;
                                weighs = (own ? above[b] : other_above[b]) >> bit & 1;
                            }
#pragma unroll
                        for (int c = 0; c < F::kColumns; ++c)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int d = 32 * c + 8 * (i / 4) + 4 * half + (i & 3);
                                if (d >= a.c.D) continue;
                                float v = pwlq_block::widen(((const C *)a.c.values)[n * a.c.D + d]);
                                if constexpr (F::kCodes) v = (float)(T)(v * a.c.value_step[n]);
                                if (!(fabsf(v) < INFINITY) && sees_it) acc[c][i] += (weighs ? 1.0f : 0.0f) * v;
                            }
                    }
                }
            }
            if (u + 1 < end) put(from + F::kKeys, at ^ 1);
            __syncthreads();
        }

        sum += __shfl_xor(sum, 32);
        if (row < t.rows) {
            const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int64_t at = (int64_t)sums * F::kRows + 32 * wave + (lane & 31);
            if (sums >= 0 && half == 0) a.top_sum[at] = make_float2(top, sum);
#pragma unroll
            for (int c = 0; c < F::kColumns; ++c)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int d = 32 * c + 2 * i + 4 * half;
                    v4f v = {acc[c][i], acc[c][i + 1], acc[c][i + 2], acc[c][i + 3]};
                    if (d >= a.c.D) continue;
                    if (sums >= 0) *(v4f *)(a.sums + at * DP + d) = v;
                    else store4<T>(a.out + ((t.q.start + j) * a.out_stride + h * a.out_head + d) * 2, sum == 0.0f ? v4f{} : v * over);
                }
        }
        __syncthreads();
    }
}

} // namespace pwlq_attention
