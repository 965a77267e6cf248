// Rows of activations in registers: element types, vectors of eight, and a row shared out among the threads of a
// workgroup.  Used by the packing, norm and adapter kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

namespace pwlq_block {

typedef __bf16 bf16;
typedef _Float16 f16;

// Vectors are as aligned as the loads need, 16 bytes at most.
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v8f __attribute__((ext_vector_type(8), aligned(16)));
typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

template <typename T> struct Vec8;
template <> struct Vec8<float> { typedef v8f type; };
template <> struct Vec8<bf16> { typedef v8bf type; };
template <> struct Vec8<f16> { typedef v8h type; };
template <> struct Vec8<int8_t> { typedef v2u type; };

// The same vectors anywhere in memory: loads and stores need the alignment of an element only (unaligned access mode), so rows
// of any length and stride move in vectors.
template <typename T> struct Loose8;
template <> struct Loose8<float> { typedef float type __attribute__((ext_vector_type(8), aligned(4))); };
template <> struct Loose8<bf16> { typedef bf16 type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct Loose8<f16> { typedef f16 type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct Loose8<int8_t> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(1))); };
template <typename T> __device__ inline typename Vec8<T>::type load8(const T *p) { return *(const typename Loose8<T>::type *)p; }
template <typename T> __device__ inline void store8(T *p, typename Vec8<T>::type v) { *(typename Loose8<T>::type *)p = v; }

__device__ inline v8f widen(v8f v) { return v; }
__device__ inline v8f widen(v8bf v) { return __builtin_convertvector(v, v8f); }
__device__ inline v8f widen(v8h v) { return __builtin_convertvector(v, v8f); }
__device__ inline v8f widen(v2u v)
{
    v8f r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (float)((int)(v[i / 4] << (24 - 8 * (i & 3))) >> 24);
    return r;
}
__device__ inline float widen(float v) { return v; }
__device__ inline float widen(bf16 v) { return (float)v; }
__device__ inline float widen(f16 v) { return (float)v; }
__device__ inline float widen(int8_t v) { return (float)v; }

// A row, or neighbouring rows, as a buffer of their own length: reads beyond its end give 0 and writes there do nothing, by the
// hardware's bounds check, so threads past the end need no branch and no select.  `row` is the same for the whole wavefront.
__device__ inline __amdgpu_buffer_rsrc_t row_buffer(const void *row, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)row, 0, (int)bytes, 0x00027000);
}
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
// Offsets in bytes.
template <typename T> __device__ inline typename Vec8<T>::type buffer_load8(__amdgpu_buffer_rsrc_t b, int offset)
{
    union { v4u w[sizeof(T) == 4 ? 2 : 1]; v2u half; typename Vec8<T>::type v; } u;
    if constexpr (sizeof(T) == 1) u.half = __builtin_amdgcn_raw_buffer_load_b64(b, offset, 0, 0);
    else u.w[0] = __builtin_amdgcn_raw_buffer_load_b128(b, offset, 0, 0);
    if constexpr (sizeof(T) == 4) u.w[1] = __builtin_amdgcn_raw_buffer_load_b128(b, offset + 16, 0, 0);
    return u.v;
}
template <typename T> __device__ inline void buffer_store8(__amdgpu_buffer_rsrc_t b, int offset, typename Vec8<T>::type v)
{
    union { v4u w[sizeof(T) == 4 ? 2 : 1]; v2u half; typename Vec8<T>::type v; } u;
    u.v = v;
    if constexpr (sizeof(T) == 1) __builtin_amdgcn_raw_buffer_store_b64(u.half, b, offset, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(u.w[0], b, offset, 0, 0);
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b128(u.w[1], b, offset + 16, 0, 0);
}
template <typename T> __device__ inline T buffer_load1(__amdgpu_buffer_rsrc_t b, int offset)
{
    union { uint32_t w; uint16_t h; uint8_t c; T v; } u;
    if constexpr (sizeof(T) == 1) u.c = __builtin_amdgcn_raw_buffer_load_b8(b, offset, 0, 0);
    else if constexpr (sizeof(T) == 2) u.h = __builtin_amdgcn_raw_buffer_load_b16(b, offset, 0, 0);
    else u.w = __builtin_amdgcn_raw_buffer_load_b32(b, offset, 0, 0);
    return u.v;
}
template <typename T> __device__ inline void buffer_store1(__amdgpu_buffer_rsrc_t b, int offset, T v)
{
    union { uint32_t w; uint16_t h; uint8_t c; T v; } u;
    u.v = v;
    if constexpr (sizeof(T) == 1) __builtin_amdgcn_raw_buffer_store_b8(u.c, b, offset, 0, 0);
    else if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(u.h, b, offset, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(u.w, b, offset, 0, 0);
}

// How the columns of a row are shared out: thread `thread` of `threads` takes E of them.
//   kSingly   single columns, as many apart as there are threads: rows of any length
//   kWhole    vectors of eight, as many vectors apart as there are threads: rows of whole vectors
//   kTail     the same where the row's last vector would pass its end: it ends there instead, and of its columns those that belong
//             to the vector before are 0 in its thread, so they add nothing to a sum or a maximum, and are not stored
// All coalesce, and rows may begin anywhere (unaligned access mode).
enum Share { kSingly, kWhole, kTail };
struct Place {
    int cols, threads, thread;
    __device__ int vector(int j) const { return (j * threads + thread) * 8; }
    __device__ int skip(int j) const { return vector(j) < cols ? max(vector(j) + 8 - cols, 0) : 0; }
    template <Share S> __device__ int start(int j) const { return S == kTail ? vector(j) - skip(j) : vector(j); }
};

// load() only reads, so several rows can be under way; get() widens.
template <typename T, int E, Share S> struct Row {
    typename std::conditional<S != kSingly, typename Vec8<T>::type, T>::type raw[S != kSingly ? E / 8 : E];

    __device__ void load(const T *row, Place at)
    {
        const __amdgpu_buffer_rsrc_t b = row_buffer(row, at.cols * (int)sizeof(T));
        if constexpr (S != kSingly) {
#pragma unroll
            for (int j = 0; j < E / 8; ++j) raw[j] = buffer_load8<T>(b, at.start<S>(j) * (int)sizeof(T));
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) raw[i] = buffer_load1<T>(b, (i * at.threads + at.thread) * (int)sizeof(T));
        }
    }
    __device__ void get(float (&v)[E], Place at) const
    {
        if constexpr (S != kSingly) {
#pragma unroll
            for (int j = 0; j < E / 8; ++j) {
                const v8f w = widen(raw[j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * j + i] = w[i];
                if (S == kTail && __ballot(at.skip(j) != 0)) {       // one wavefront's
#pragma unroll
                    for (int i = 0; i < 7; ++i) v[8 * j + i] = i < at.skip(j) ? 0.0f : w[i];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = widen(raw[i]);
        }
    }
};

// Nothing is moved across: the loads above it are issued before what uses them.  The compiler would otherwise put each beside its use,
// which saves registers and waits for memory once per load.
__device__ inline void loads_first() { __builtin_amdgcn_sched_barrier(0); }

// A vector of a row: all of it, or its own columns one by one.
template <typename T, Share S> __device__ inline void store_vector(__amdgpu_buffer_rsrc_t b, Place at, int j, typename Vec8<T>::type v)
{
    const int skip = S == kTail ? at.skip(j) : 0;
    if (skip == 0) buffer_store8<T>(b, at.vector(j) * (int)sizeof(T), v);
    else {
        union { typename Vec8<T>::type v; T e[8]; } u;
        u.v = v;
#pragma unroll
        for (int i = 1; i < 8; ++i)
            if (i >= skip) buffer_store1<T>(b, (at.vector(j) - skip + i) * (int)sizeof(T), u.e[i]);
    }
}
template <typename T, int E, Share S> __device__ inline void store_row(T *row, Place at, const float (&v)[E])
{
    const __amdgpu_buffer_rsrc_t b = row_buffer(row, at.cols * (int)sizeof(T));
    if constexpr (S != kSingly) {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            v8f w;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = v[8 * j + i];
            store_vector<T, S>(b, at, j, __builtin_convertvector(w, typename Vec8<T>::type));
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) buffer_store1<T>(b, (i * at.threads + at.thread) * (int)sizeof(T), (T)v[i]);
    }
}

// Sum, or maximum of unsigned words, over a wavefront: a scan along each row of sixteen lanes, then along the rows, all by
// data-parallel moves; the last lane has the result.  0 is neutral for both.
template <int CONTROL, int ROWS> __device__ inline uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, ROWS, 0xf, true);
}
__device__ inline float wave_sum(float v)
{
#define PWLQ_STEP(CONTROL, ROWS) v += __uint_as_float(moved<CONTROL, ROWS>(__float_as_uint(v)))
    PWLQ_STEP(0x111, 0xf);             // one lane up
    PWLQ_STEP(0x112, 0xf);
    PWLQ_STEP(0x114, 0xf);
    PWLQ_STEP(0x118, 0xf);
    PWLQ_STEP(0x142, 0xa);             // a row's last lane to the next row
    PWLQ_STEP(0x143, 0xc);             // lane 31 to the upper half
#undef PWLQ_STEP
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}
__device__ inline uint32_t wave_max(uint32_t v)
{
#define PWLQ_STEP(CONTROL, ROWS) v = max(v, moved<CONTROL, ROWS>(v))
    PWLQ_STEP(0x111, 0xf);
    PWLQ_STEP(0x112, 0xf);
    PWLQ_STEP(0x114, 0xf);
    PWLQ_STEP(0x118, 0xf);
    PWLQ_STEP(0x142, 0xa);
    PWLQ_STEP(0x143, 0xc);
#undef PWLQ_STEP
    return __builtin_amdgcn_readlane(v, 63);
}

// The same over a workgroup of whole wavefronts, at most 16.  `slots`: LDS of this reduction alone, a word per wavefront (two for
// two sums), not written again before the workgroup's next barrier.  Every thread gets the same result, and the order is fixed.
__device__ inline float block_sum(float v, float *slots, int threads)
{
    v = wave_sum(v);
    if (threads == 64) return v;
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < threads / 64; ++w) s += slots[w];
    return s;
}
__device__ inline void block_sum2(float &v, float &u, float2 *slots, int threads)
{
    v = wave_sum(v);
    u = wave_sum(u);
    if (threads == 64) return;
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = make_float2(v, u);
    __syncthreads();
    v = u = 0.0f;
    for (int w = 0; w < threads / 64; ++w) {
        v += slots[w].x;
        u += slots[w].y;
    }
}
__device__ inline uint32_t block_max(uint32_t v, uint32_t *slots, int threads)
{
    v = wave_max(v);
    if (threads == 64) return v;
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t s = 0;
    for (int w = 0; w < threads / 64; ++w) s = max(s, slots[w]);
    return s;
}

// Step and factor of a row whose largest magnitude has these bits.  As unsigned words the bits of magnitudes are in the
// order of their values, infinities next and NaN above, so one maximum finds all three.
struct Step { float step, factor; };
constexpr uint32_t kInfinityBits = 0x7f800000u, kLeastBits = (127u - 100u) << 23;     // 2^-100
__device__ inline Step step_of(uint32_t bits)
{
    Step s = {0.0f, 0.0f};
    const float a = __uint_as_float(bits);
    if (bits >= kInfinityBits) s.step = __uint_as_float(0x7fc00000u);
    else if (bits >= kLeastBits) {
        s.step = a / 127.0f;
        s.factor = 127.0f / a;
    }
    return s;
}
template <int E> __device__ inline uint32_t largest(const float (&v)[E])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E; i += 2) m = max(max(m, __float_as_uint(v[i]) & 0x7fffffffu), __float_as_uint(v[i + 1]) & 0x7fffffffu);
    return m;
}

// rne(x factor) in the low byte: added to 1.5 2^23 the product's fraction is rounded away.  |x factor| is at most 127.
__device__ inline uint32_t code_byte(float x, float factor) { return __float_as_uint(x * factor + 12582912.0f); }
__device__ inline uint32_t four_codes(const float *x, float factor)
{
    const uint32_t a = __builtin_amdgcn_perm(code_byte(x[1], factor), code_byte(x[0], factor), 0x0c0c0400u);
    const uint32_t b = __builtin_amdgcn_perm(code_byte(x[3], factor), code_byte(x[2], factor), 0x0c0c0400u);
    return __builtin_amdgcn_perm(b, a, 0x05040100u);
}

// Codes of a row.  With factor 0 (a row of next to nothing, or one that holds a NaN or an infinity) all are 0, whatever v is.
template <int E, Share S> __device__ inline void store_codes(int8_t *row, Place at, const float (&v)[E], float factor)
{
    const __amdgpu_buffer_rsrc_t b = row_buffer(row, at.cols);
    const bool none = factor == 0.0f;
    if constexpr (S != kSingly) {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            v2u q = {0u, 0u};
            if (!none) q = v2u{four_codes(v + 8 * j, factor), four_codes(v + 8 * j + 4, factor)};
            store_vector<int8_t, S>(b, at, j, q);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) buffer_store1<int8_t>(b, i * at.threads + at.thread, none ? 0 : (int8_t)code_byte(v[i], factor));
    }
}

} // namespace pwlq_block
