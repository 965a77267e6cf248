// k_pack_rows: rows of activations to 8 bits with a step each.  k_unpack_rows: the values they stand for.
//
//   a = max|x|,  step = a/127,  code = rne(x * (127/a))
// The codes are the operand of the integer inner product (its s_x is 1: the step is a factor of the output row) and
// the activation checkpoint of a backward pass, at half the bytes of bfloat16 or a quarter of binary32's.
//
// Both are bound by memory.  A row is read once: it stays in its workgroup's registers between the maximum and
// the rounding.  4096 x 11008 of bfloat16: packed in 24 us (135 MB, 5.6 TB/s), unpacked in 21 (6.5 TB/s, the codes partly still in
// the last-level cache); 515 x 1155 of binary32 3.2 and 2.9 us, which is a launch.
#include "launch.h"
#include "rows.h"

namespace pwlq_block {
namespace {

template <typename T, int E, Share S>
__global__ __launch_bounds__(1024) void k_pack_rows(const T *x, int64_t stride, int64_t rows, int cols, int8_t *codes, float *step)
{
    __shared__ uint32_t slots[2][16];
    const int threads = blockDim.x, thread = threadIdx.x;
    const Place at = {cols, threads, thread};
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        Row<T, E, S> r;
        float v[E];
        r.load(x + row * stride, at);
        r.get(v, at);
        const Step s = step_of(block_max(largest(v), slots[turn], threads));
        store_codes<E, S>(codes + row * cols, at, v, s.factor);
        if (thread == 0) step[row] = s.step;
    }
}

template <typename T, int E, Share S>
__global__ __launch_bounds__(1024) void k_unpack_rows(const int8_t *codes, const float *step, int64_t rows, int cols, T *out, int64_t stride)
{
    const int threads = blockDim.x, thread = threadIdx.x;
    const Place at = {cols, threads, thread};
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        Row<int8_t, E, S> r;
        float v[E];
        r.load(codes + row * cols, at);
        r.get(v, at);
        const float s = step[row];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] *= s;
        store_row<T, E, S>(out + row * stride, at, v);
    }
}

inline int threads_for(int cols, int E) { return (cols + 64 * E - 1) / (64 * E) * 64; }

// Elements of a thread: 16 up to 16384 columns (a workgroup holds 1024 threads), else what the longest rows need: 2048 x 32768 of
// bfloat16 31 us packed and 31 unpacked (6.5 TB/s), of binary32 64 and 82.  Where single columns are moved that spills 8 to 29 registers:
// 4096 x 16388 of bfloat16 102 and 44, 4096 x 16384 31 and 30 (replayed, inputs partly in the last-level cache).
template <typename T, Share S>
void pack_as(const pwlq_rows &x, int64_t rows, int K, int8_t *codes, float *step, hipStream_t stream)
{
    const unsigned grid = row_grid(rows);
#define PWLQ_PACK(E) \
    k_pack_rows<T, E, S><<<grid, threads_for(K, E), 0, stream>>>((const T *)x.data, x.stride, rows, K, codes, step)
    if (K <= 512) PWLQ_PACK(8);
    else if (K <= 16384) PWLQ_PACK(16);
    else PWLQ_PACK(64);
#undef PWLQ_PACK
}

template <typename T, Share S>
void unpack_as(const int8_t *codes, const float *step, int64_t rows, int K, const pwlq_rows &out, hipStream_t stream)
{
    const unsigned grid = row_grid(rows);
#define PWLQ_UNPACK(E) \
    k_unpack_rows<T, E, S><<<grid, threads_for(K, E), 0, stream>>>(codes, step, rows, K, (T *)out.data, out.stride)
    if (K <= 512) PWLQ_UNPACK(8);
    else if (K <= 16384) PWLQ_UNPACK(16);
    else PWLQ_UNPACK(64);
#undef PWLQ_UNPACK
}

} // namespace

void pack_rows(const pwlq_rows &x, int64_t rows, int K, int8_t *codes, float *step, hipStream_t stream)
{
    // rows of no whole vectors singly: 2000 x 4091 of bfloat16, packed and unpacked, 13.0 us; in vectors, the last one apart, 14.5
#define PWLQ_AS(T) (K % 8 == 0 ? pack_as<T, kWhole>(x, rows, K, codes, step, stream) : pack_as<T, kSingly>(x, rows, K, codes, step, stream))
    if (x.type == PWLQ_F32) PWLQ_AS(float);
    else if (x.type == PWLQ_BF16) PWLQ_AS(bf16);
    else PWLQ_AS(f16);
#undef PWLQ_AS
}

void unpack_rows(const int8_t *codes, const float *step, int64_t rows, int K, const pwlq_rows &out, hipStream_t stream)
{
#define PWLQ_AS(T) \
    (K % 8 == 0 ? unpack_as<T, kWhole>(codes, step, rows, K, out, stream) : unpack_as<T, kSingly>(codes, step, rows, K, out, stream))
    if (out.type == PWLQ_F32) PWLQ_AS(float);
    else if (out.type == PWLQ_BF16) PWLQ_AS(bf16);
    else PWLQ_AS(f16);
#undef PWLQ_AS
}

} // namespace pwlq_block
