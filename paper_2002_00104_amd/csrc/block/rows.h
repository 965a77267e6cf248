// Rows of activations in registers: element types, vectors of eight, and a row shared out among the threads of a
// workgroup.  Used by the packing, norm and adapter kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

template <typename T> __device__ inline v8f load8(const T *p) { return widen(*(const typename Vec8<T>::type *)p); }
template <typename T> __device__ inline void store8(T *p, v8f v)
{
    *(typename Vec8<T>::type *)p = __builtin_convertvector(v, typename Vec8<T>::type);
}

// Eight codes in two words; a code is a whole number within +-127 held in binary32.
__device__ inline v2u codes8(v8f q)
{
    v2u r = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i / 4] |= ((uint32_t)(int)q[i] & 0xffu) << (8 * (i & 3));
    return r;
}

// Column of a thread's element i.  VEC: vectors of eight columns, as many vectors apart as there are threads; else
// single columns that far apart.  Both coalesce, the second for any length and alignment.
template <bool VEC> __device__ inline int column(int i, int threads, int thread)
{
    return VEC ? ((i >> 3) * threads + thread) * 8 + (i & 7) : i * threads + thread;
}

// Columns of one row: thread `thread` of `threads` takes E.  Those past the row's end are 0.
template <typename T, int E, bool VEC>
__device__ inline void load_row(const T *row, int cols, int threads, int thread, float (&v)[E])
{
    if constexpr (VEC) {
        typename Vec8<T>::type raw[E / 8];
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            const int c = (j * threads + thread) * 8;
            raw[j] = c < cols ? *(const typename Vec8<T>::type *)(row + c) : typename Vec8<T>::type(0);
        }
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            const v8f w = widen(raw[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * j + i] = w[i];
        }
    } else {
        T raw[E];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = i * threads + thread;
            raw[i] = c < cols ? row[c] : T(0);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = widen(raw[i]);
    }
}

template <typename T, int E, bool VEC>
__device__ inline void store_row(T *row, int cols, int threads, int thread, const float (&v)[E])
{
    if constexpr (VEC) {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            const int c = (j * threads + thread) * 8;
            v8f w;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = v[8 * j + i];
            if (c < cols) store8(row + c, w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = i * threads + thread;
            if (c < cols) row[c] = (T)v[i];
        }
    }
}

// Sum, or maximum of unsigned words, over a workgroup of whole wavefronts.  `slots`: LDS of this reduction alone, a word
// per wavefront (at most 16), not written again before the workgroup's next barrier.  Every thread gets the same result: the
// order of the sum is fixed.
__device__ inline float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ inline uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    return v;
}
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
// With factor 0 the code is 0 whatever the element is: rows that hold a NaN or an infinity.
__device__ inline float code_of(float x, float factor) { return factor == 0.0f ? 0.0f : __builtin_rintf(x * factor); }

template <int E> __device__ inline uint32_t largest(const float (&v)[E])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}

template <int E, bool VEC>
__device__ inline void store_codes(int8_t *row, int cols, int threads, int thread, const float (&v)[E], float factor)
{
    if constexpr (VEC) {
#pragma unroll
        for (int j = 0; j < E / 8; ++j) {
            const int c = (j * threads + thread) * 8;
            v8f q;
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = code_of(v[8 * j + i], factor);
            if (c < cols) *(v2u *)(row + c) = codes8(q);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = i * threads + thread;
            if (c < cols) row[c] = (int8_t)(int)code_of(v[i], factor);
        }
    }
}

} // namespace pwlq_block
