// k_attend_many: tiles of 128 query rows, for prompts and larger trees.
//
// Bound by the matrix cores and by the exponentials beside them, one after the other: a tile of 64 keys takes a wavefront's 32 rows 1024 cycles of matrix
// instructions (128 channels) and nearly as many of vector instructions for its 2048 weights.  Two workgroups share a CU, but one's products run
// beside the other's exponentials by chance only: a prompt of 4096 rows, 32 heads over 8, takes 160 us, 860 TFLOP/s, with the matrix cores
// busy in 47 % of the cycles and vector instructions issued in as many others.  1024 rows after 7169 in 8 bits, capped: 237 us with the join, 553 TFLOP/s, 25 and
// 60 %: codes and caps are vector instructions.
//
// Keys and values of a tile are staged in LDS, twice: one is filled while the other is worked on, a barrier a tile; 16-bit elements
// go there from memory directly, codes too, and are widened there between two barriers.  As for few
// rows, S^T = K Q^T leaves a lane its query row's weights in the layout of the operand of O^T = V^T P^T.
#pragma once

#include "attend.h"

namespace pwlq_attention {

// DP: channels that a row in LDS has room for, DC: those that are multiplied, no fewer than D.
template <typename T, typename C, int DP, int DC> struct Many {
    static constexpr bool kCodes = sizeof(C) == 1, kScaled = kCodes && __is_same(T, f16);    // values scaled as they are read
    static constexpr bool kMayBeBad = !kCodes || kScaled;                          // values that are not finite
    static constexpr int kRows = 128, kKeys = DP == 256 ? 32 : 64;                 // of a unit; a wavefront has 32 rows
    static constexpr int kSteps = DC / 16, kColumns = DC / 32, kBlocks = kKeys / 32;
    static constexpr int kChunks = kCodes ? DP / 16 : DP / 8;                      // of 16 bytes, of a row in memory
    static constexpr int kPass = 256 / kChunks, kLoads = kKeys / kPass, kWavePass = 64 / kChunks;
    static constexpr int kTurns = kPass % 16 ? 16 / kPass : 1;                     // loads after which rows lie in a block as at first
    static constexpr int kAhead = 8;                                               // operands of keys under way
    // In LDS, a stage: keys, then values.  16-bit elements have two; codes one, and then codes of keys and of values as they come.
    static constexpr int kRowBytes = 2 * DP, kPart = kKeys * kRowBytes, kStage = 2 * kPart, kCodePart = kKeys * DP;
    static constexpr int kRoom = kCodes ? kStage + 2 * kCodePart : 2 * kStage;
    static_assert(kRoom >= kPlanBytes, "LDS");
    typedef typename Vec8<T>::type v8;

    // A row's chunks of 16 bytes in LDS are in an order of its own, so that the rows that are read together lie in different banks: for keys
    // sixteen rows' chunks of one number, for values four rows' chunks of four numbers.
    static __device__ int key_swizzle(int row) { return DP == 64 ? (row >> 1) & 7 : row & 15; }
    static __device__ int value_swizzle(int row) { return DP == 64 ? 4 * ((row >> 1) & 1) : 4 * (row & 3); }

    float step;                                                                    // of codes: a key's or a value's, by the wavefront

    // What a lane fetches of a pass's rows, in bytes from their block's first row: of keys and of values.  It goes to LDS by itself, where a
    // wavefront fills whole rows one after the other: the lane that fills a chunk fetches what belongs there.  Negative: nothing, past D.
    int key_from[kTurns], value_from[kTurns];
    __device__ void prepare(const Attend &a, int wave, int lane)
    {
        const int D = a.c.D, chunk = lane % kChunks;
#pragma unroll
        for (int j = 0; j < kTurns; ++j) {
            const int row = (j * kPass + wave * kWavePass) % 16 + lane / kChunks;
            if constexpr (kCodes) {
                key_from[j] = value_from[j] = chunk * 16 < D ? row * D + chunk * 16 : -1;
            } else {
                const int of_key = 8 * (chunk ^ key_swizzle(row)), of_value = 8 * (chunk ^ value_swizzle(row));
                key_from[j] = of_key < D ? 2 * (row * D + of_key) : -1;
                value_from[j] = of_value < D ? 2 * (row * D + of_value) : -1;
            }
        }
    }
    // A unit's keys and values to LDS, codes as they are.  Its blocks are those of lane `block` on, `rows` the number of the first row of each.
    __device__ void load(const Attend &a, char *room, int64_t rows, int block, int wave, int lane)
    {
        const int64_t bytes = rows * (a.c.D * (int)sizeof(C));                     // of every lane's block, of which one is taken
        constexpr int kLine = kCodes ? DP : kRowBytes, kValues = kCodes ? kCodePart : kPart;
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)room + (kCodes ? kStage : 0) + wave * kWavePass * kLine;
        int64_t at[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int from = block + (j * kPass + wave * kWavePass) / 16;
            at[j] = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)bytes, from) |
                              (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(bytes >> 32), from) << 32);
        }
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            if (key_from[turn] >= 0) {
#pragma unroll
                for (int j = turn; j < kLoads; j += kTurns) to_lds(a.c.keys + at[j], (uint32_t)key_from[turn], to + j * kPass * kLine);
            }
            if (value_from[turn] >= 0) {
#pragma unroll
                for (int j = turn; j < kLoads; j += kTurns) to_lds(a.c.values + at[j], (uint32_t)value_from[turn], to + j * kPass * kLine + kValues);
            }
        }
        if constexpr (kCodes) {
            // by all lanes: the blocks' rows may be in lanes that have no step to fetch, and a lane that is off gives 0
            const int of = (block + lane / 16) & 63;
            const int64_t n = (int64_t)((uint64_t)(uint32_t)__shfl((int)rows, of) | (uint64_t)(uint32_t)__shfl((int)(rows >> 32), of) << 32);
            if (wave < 2 && lane < kKeys) step = (wave ? a.c.value_step : a.c.key_step)[n + (lane & 15)];
        }
    }
    // Sixteen bytes for each lane, to LDS from `to` on in the order of the lanes.  Written out, since the compiler takes what comes to LDS this way to
    // come to all of it and would wait before every read of the other buffer; the wait is in arrive().  It writes no register; m0, which says where to, is
    // an operand.  Five wait states come before it, which the compiler does not count here: a scalar register that a vector instruction has written
    // (readlane, of a scalar that was spilled too) may be read as an address then.
    static __device__ void to_lds(const char *from, uint32_t offset, uint32_t to)
    {
        // the same in all lanes, said so for what is compiled with less analysis
        const uint32_t place = __builtin_amdgcn_readfirstlane((int)to);
        const uint64_t address = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint64_t)from) |
                                 (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)from >> 32)) << 32;
        asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(place), "v"(offset), "s"(address) : "memory");
    }
    // The steps that load() fetched: keys' times what makes scores of products.
    __device__ void put_steps(float *steps, float to_score, int wave, int lane) const
    {
        if (wave < 2 && lane < kKeys) steps[wave * kKeys + lane] = wave ? step : step * to_score;
    }
    // Codes that are in LDS as T in the stage.  `checked`: some row does not see all keys, see Few::put_values.
    static __device__ bool widen_codes(const Attend &a, char *room, const float *steps, bool checked, int from, int end, uint32_t none)
    {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = j * 256 + threadIdx.x, r = i / kChunks, chunk = i % kChunks;
            const v4u k = ((const v4u *)(room + kStage))[i], v = ((const v4u *)(room + kStage + kCodePart))[i];
            float step = 0.0f;
            if (kScaled && !(checked && (from + r >= end || (none >> (r / 16) & 1)))) step = steps[kKeys + r];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                *(v4u *)(room + r * kRowBytes + 16 * ((2 * chunk + h) ^ key_swizzle(r))) = words<T>(codes8<T>(k[2 * h], k[2 * h + 1]));
                v4u w;
                if constexpr (kScaled) {
                    w = words<T>(codes8<T>(v[2 * h], v[2 * h + 1], step));
                    if (checked) bad |= make_finite<T>(w) && chunk * 16 < a.c.D;
                } else {
                    w = words<T>(codes8<T>(v[2 * h], v[2 * h + 1]));
                }
                *(v4u *)(room + kPart + r * kRowBytes + 16 * ((2 * chunk + h) ^ value_swizzle(r))) = w;
            }
        }
        return __ballot(bad) != 0;
    }
    // 16-bit values that are in LDS, of a tile of which some row does not see all keys.  `none`: blocks without a page.
    __device__ static bool check(const Attend &a, char *room, int from, int end, uint32_t none)
    {
        bool bad = false;
#pragma unroll 1
        for (int i = threadIdx.x; i < kPart / 16; i += 256) {
            const int r = i / (DP / 8), chunk = (i % (DP / 8)) ^ value_swizzle(r);
            v4u *const at = (v4u *)(room + kPart) + i;
            v4u w = *at;
            if (from + r >= end || (none >> (r / 16) & 1)) w = v4u{0u, 0u, 0u, 0u};
            bad |= make_finite<T>(w) && 8 * chunk < a.c.D;
            *at = w;
        }
        return __ballot(bad) != 0;
    }
};

template <typename T, typename C, int DP, int DC, Scores SCORES>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attend_many(const Attend a)
{
    typedef Many<T, C, DP, DC> F;
    typedef typename F::v8 v8;
    __shared__ __attribute__((aligned(16))) char room[F::kRoom];
    __shared__ __attribute__((aligned(16))) float steps[2][F::kCodes ? 2 * F::kKeys : 4];   // read four at a time; of the unit that is worked on, and of the next
    __shared__ int bad;                                    // a value taken out
    __shared__ Tile tiles[kFewTiles];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const float to_cap = SCORES == kCapped ? a.scale / a.cap : a.scale * kLog2e, cap2 = a.cap * kLog2e;
    // Plain scores stay as the product has them until the exponential, whose addition takes the factor too.  Where the scale is negative the
    // queries change their sign; it is not 0 here, which times what is masked would be NaN.
    const float factor = SCORES == kPlain ? fabsf(to_cap) : 1.0f;

    Segments<F::kRows, F::kKeys, 256> segments(a, (uint32_t *)room, tiles);
    if (a.c.D != DP) {
        // channels past D, which nothing is fetched to
        for (int i = threadIdx.x; i < F::kRoom / 16; i += 256) ((v4u *)room)[i] = v4u{0u, 0u, 0u, 0u};
        __syncthreads();
    }
    F f;
    f.prepare(a, wave, lane);
    while (segments.next(a)) {
        const Tile t = segments.t;
        const int head = segments.head, sums = segments.sums;
        const int32_t *const table = a.b.table + t.s * a.b.table_stride;
        const int begin = segments.begin, end = min(segments.stop, (t.hi + F::kKeys - 1) / F::kKeys);
        int64_t rows = 0;                                  // lane i: the first row of block base + i of sixteen keys,
        uint64_t missing = 0;                              // bit i: which has no page
        int base = 0;
        auto load = [&](int u, int to) {
            const int block = u * (F::kKeys / 16);
            if (u == begin || block - base == 64) {
                base = block;
                const int slot = 16 * (base + lane);
                int page = -1;
                if (slot < t.hi) {
                    page = table[slot >> a.c.shift];
                    if ((unsigned)page >= (unsigned)a.c.pages) page = -1;
                }
                missing = __ballot(page < 0);
                rows = row_number(a.c, Place{max(page, 0), slot & ((1 << a.c.shift) - 1)}, head);
            }
            f.load(a, room + to * F::kStage, rows, block - base, wave, lane);
        };
        if (threadIdx.x == 0) bad = 0;
        if (begin < end) load(begin, 0);
        // the queries and masks while the first keys are on their way
        const int row = t.first + 32 * wave + (lane & 31), clamped = min(row, t.rows - 1);
        const RowState state = row_state(a, t, row, head);
        const int j = by_group(a, clamped), h = head * a.group + clamped - j * a.group;
        const T *const in = (const T *)a.q + (int64_t)(t.q.start + j) * a.q_stride + h * a.q_head;
        v8 q[F::kSteps];
#pragma unroll
        for (int s = 0; s < F::kSteps; ++s) {
            const int d = 16 * s + 8 * half;
            q[s] = v8{};
            if (row < t.rows && d < a.c.D) q[s] = pwlq_block::load8<T>(in + d);
            if (SCORES == kPlain && a.scale < 0.0f) q[s] = -q[s];
        }
        v16f acc[F::kColumns];
#pragma unroll
        for (int c = 0; c < F::kColumns; ++c) acc[c] = v16f{};
        float top = -INFINITY, reference = 0.0f, sum = 0.0f;
        bool far = false;                                  // some row's reference is beyond kFar

        const int last = min(t.first + F::kRows, t.rows) - 1;
        // this wavefront's rows, and the slots that any of them may see
        const int my_first = min(t.first + 32 * wave, last), my_last = min(my_first + 31, last);
        int my_end = t.hi, my_begin = t.lo;
        if (!a.tree) {
            my_end = min(max(t.q.kept() + by_group(a, my_last) + 1, t.prefix), t.hi);
            if (a.window && !t.prefix) my_begin = max(t.q.kept() + by_group(a, my_first) - a.window + 1, t.lo);
        }
        if (t.first + 32 * wave > last) my_end = 0;
        const Common whole = common(a, t, t.first, last);
        auto lacks_of = [&](int u) { return (uint32_t)(missing >> (u * (F::kKeys / 16) - base)) & ((1u << F::kKeys / 16) - 1); };
        // What was loaded last is in LDS for all wavefronts, and nobody reads the other buffer any more.
        auto arrive_whole = [&](int u) {
            __builtin_amdgcn_s_waitcnt(0x0f70);            // what was on its way to LDS: vmcnt(0)
            if constexpr (F::kCodes) {
                f.put_steps(steps[u & 1], SCORES == kPlain ? 1.0f : to_cap, wave, lane);
                __syncthreads();
                F::widen_codes(a, room, steps[u & 1], false, 0, 0, 0u);
            }
            __syncthreads();
        };
        auto arrive = [&](int u, int to) {
            const int from = u * F::kKeys;
            const uint32_t none = lacks_of(u);
            if (none == 0 && whole.has(from, from + F::kKeys)) {
                arrive_whole(u);
                return;
            }
            __builtin_amdgcn_s_waitcnt(0x0f70);
            if constexpr (F::kCodes) f.put_steps(steps[u & 1], SCORES == kPlain ? 1.0f : to_cap, wave, lane);
            __syncthreads();
            if (F::kCodes ? F::widen_codes(a, room, steps[u & 1], true, from, t.hi, none) : F::check(a, room + to * F::kStage, from, t.hi, none)) bad = 1;
            __syncthreads();
        };
        const int key_at = (lane & 31) * F::kRowBytes + 16 * (F::key_swizzle(lane & 31) ^ half);
        const int value_row = 4 * half + (lane & 15) / 4;
        const int value_at = F::kPart + value_row * F::kRowBytes + 16 * (F::value_swizzle(value_row) ^ (2 * ((lane >> 4) & 1) + (lane >> 1 & 1))) + 8 * (lane & 1);
        // A unit's work; `masked`: some row of the wavefront's may not see all keys.
        auto work = [&](int u, int at, auto masked, uint32_t none) {
            const int from = u * F::kKeys;
            // operands are read from LDS some products before they are needed
            auto key = [&](int b, int i) { return as8<T>(*(const v4u *)(room + at * F::kStage + (key_at ^ 32 * i) + b * 32 * F::kRowBytes)); };
            auto value = [&](int step, int c) {
                const char *const p = room + at * F::kStage + (value_at ^ 64 * c) + 16 * step * F::kRowBytes;
                return columns8<T>(p, p + 8 * F::kRowBytes);
            };
            v16f s[F::kBlocks];
            v8 k[F::kAhead], v[F::kColumns];
#pragma unroll
            for (int i = 0; i < F::kAhead; ++i) k[i] = key(i / F::kSteps, i % F::kSteps);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < F::kBlocks * F::kSteps; ++n) {
                const int b = n / F::kSteps, next = n + F::kAhead;
                if (n % F::kSteps == 0) s[b] = v16f{};
                s[b] = mfma32(k[n % F::kAhead], q[n % F::kSteps], s[b]);
                if (next < F::kBlocks * F::kSteps) k[n % F::kAhead] = key(next / F::kSteps, next % F::kSteps);
            }
#pragma unroll
            for (int c = 0; c < F::kColumns; ++c) v[c] = value(0, c);
            __builtin_amdgcn_sched_barrier(0);
            // element i of block b is key 32 b + 8 (i / 4) + 4 half + i % 4
#pragma unroll
            for (int b = 0; b < F::kBlocks; ++b) {
                if constexpr (F::kCodes) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const v4f w = *(const v4f *)(steps[u & 1] + 32 * b + 2 * i + 4 * half);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][i + e] *= w[e];
                    }
                }
                if constexpr (SCORES != kPlain) {
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = s[b][i];
                    if constexpr (!F::kCodes) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] *= to_cap;
                    }
                    if constexpr (SCORES == kCapped) cap_scores(x, cap2);
                    if (a.slopes) {
                        const float away = (float)(state.own - from - 32 * b - 4 * half);
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = __builtin_fmaf(-state.slope, fabsf(away - (float)(8 * (i / 4) + (i & 3))), x[i]);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = x[i];
                }
            }
            uint64_t seen = ~0ull;
            if constexpr (masked.value) {
                seen = seen_slots(a, t, state, from);
#pragma unroll
                for (int b = 0; b < F::kKeys / 16; ++b)
                    if (none >> b & 1) seen &= ~(0xffffull << (16 * b));
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b) {
                    const uint32_t of = (uint32_t)(seen >> (32 * b)) >> (4 * half);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = of >> (8 * (i / 4) + (i & 3)) & 1 ? s[b][i] : -INFINITY;
                }
            }
            float most = -INFINITY;
#pragma unroll
            for (int b = 0; b < F::kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, s[b][i]);
            most *= factor;
            if (__ballot(most > top + kSlack)) {
                most = fmaxf(top, fmaxf(most, __shfl_xor(most, 32)));
                const float next = reference_of<T>(most);
                // a sum that is NaN already stays NaN
                const float old = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(reference - next);
                sum *= old;
#pragma unroll
                for (int c = 0; c < F::kColumns; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c][i] *= old;
                top = most;
                reference = next;
                if constexpr (SCORES == kPlain) far = __ballot(fabsf(reference) >= kFar) != 0;
            }
            // The reference is a rounded product, and what that is off by is in all of a row's weights, as a factor.  Far out it would be any
            // number, so there the others are rounded products too.
            float by = factor, less = reference;
            if (SCORES == kPlain && far) {
#pragma unroll
                for (int b = 0; b < F::kBlocks; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = s[b][i] * factor - reference;
                by = 1.0f;
                less = 0.0f;
            }
            // a unit's weights are summed by themselves: one by one they might be nothing beside what there is
            float more = 0.0f;
            v8 weight[F::kBlocks][2];
#pragma unroll
            for (int b = 0; b < F::kBlocks; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], by, -less));
                    more += s[b][i];
                }
                if constexpr (F::kCodes && !F::kScaled) {
                    // a row's step joins its weight: one rounding to bfloat16, of their product; a step may be NaN
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const v4f w = *(const v4f *)(steps[u & 1] + F::kKeys + 32 * b + 2 * i + 4 * half);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][i + e] *= w[e];
                    }
                    if constexpr (masked.value) {
                        const uint32_t of = (uint32_t)(seen >> (32 * b)) >> (4 * half);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[b][i] = of >> (8 * (i / 4) + (i & 3)) & 1 ? s[b][i] : 0.0f;
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
            sum += more;
#pragma unroll
            for (int step = 0; step < 2 * F::kBlocks; ++step)
#pragma unroll
                for (int c = 0; c < F::kColumns; ++c) {
                    acc[c] = mfma32(v[c], weight[step / 2][step & 1], acc[c]);
                    if (step + 1 < 2 * F::kBlocks) v[c] = value(step + 1, c);
                }
        };
        __syncthreads();
        if (begin < end) arrive(begin, 0);
        // Units that all rows see whole, as they mostly are, have a loop of their own, with nothing about masks in it.
        constexpr int kOther = F::kCodes ? 0 : 1;          // of two stages the one that is filled
        int u = begin, at = 0;
        auto whole_to = [&](int u) {                       // the end of such units from u on, none of which lacks a page
            const int from = u * F::kKeys;
            int stop = u;
            if (whole.has(from, from + F::kKeys)) stop = max(from >= whole.begin ? whole.end : 0, whole.prefix) / F::kKeys;
            stop = min(stop, end);
            const uint64_t holes = missing >> (u * (F::kKeys / 16) - base);
            // as far as the pages are known that are there
            return min(stop, u + min((int)__builtin_ctzll(holes | 1ull << 63), 64 - (u * (F::kKeys / 16) - base)) / (F::kKeys / 16));
        };
        const bool mine = t.first + 32 * wave <= last;
        while (u < end) {
            for (const int stop = whole_to(u) - 1; u < stop; ++u, at ^= kOther) {
                load(u + 1, at ^ kOther);
                if (mine) work(u, at, std::false_type(), 0u);
                arrive_whole(u + 1);
            }
            const uint32_t none = lacks_of(u);
            const int from = u * F::kKeys;
            if (u + 1 < end) load(u + 1, at ^ kOther);
            if (from < my_end && from + F::kKeys > my_begin) work(u, at, std::true_type(), none);
            if (u + 1 < end) arrive(u + 1, at ^ kOther);
            ++u;
            at ^= kOther;
        }

        if (F::kMayBeBad && __builtin_amdgcn_readfirstlane(bad)) {
#pragma unroll
            for (int c = 0; c < F::kColumns; ++c) {
                v16f count = {}, sign = {};
                for (int from = begin * F::kKeys; from < end * F::kKeys; from += 16) {
                    const uint32_t mine = (uint32_t)(seen_slots(a, t, state, from) >> (4 * half));
                    const NotFinite<T, C> v(a, table, head, from + 4 * half, 8, t.hi, 32 * c + (lane & 31), (mine & 15) | (mine >> 4 & 0xf0));
                    count = mfma32(v.counts, v.ones, count);
                    sign = mfma32(v.signs, v.ones, sign);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[c][i] += not_finite_sum(count[i], sign[i]);
            }
        }
        sum += __shfl_xor(sum, 32);
        if (row < t.rows) {
            const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
            const int64_t at = (int64_t)sums * F::kRows + 32 * wave + (lane & 31);
            if (sums >= 0 && half == 0) a.top_sum[at] = make_float2(top == -INFINITY ? top : reference, sum);
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
