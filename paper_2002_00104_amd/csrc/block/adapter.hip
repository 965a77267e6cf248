// Low-rank adapters of many requests beside a shared projection, and their gradients.  Three products carry both directions,
// for matrices W [adapters, R, C] with the rank before the columns, and the rows t of a batch with adapter a(t):
//   first   H[t] = scale[a] X[t] W[a]^T             (forward: x, down; backward: dy, up)
//   second  Y[t] = base[t] + H[t] W[a]              (forward: h, up; backward: dh, down)
//   outer   G[a] = sum over its rows of H[t] (x) X[t]       (d_down: dh, x; d_up: h, dy)
// With ranks of 16 to 64 all three are bound by memory: per element of X or Y they do 2 R operations.
//
// Rows of one request are next to each other, so most tiles of rows have one adapter; a tile of several is done once for
// each, and a row keeps what its own adapter gave: nothing is sorted, and any order of ids is right.
#include <algorithm>

#include "launch.h"
#include "rows.h"

#pragma clang fp contract(fast)

namespace pwlq_block {
namespace {

constexpr int kRows = 32;              // rows of a tile of the first product: two of the matrix instructions'

// Nothing is moved across: the loads above it are issued before what uses them.  The compiler would otherwise put each beside its use,
// which saves registers and waits for memory once per load.
__device__ inline void loads_first() { __builtin_amdgcn_sched_barrier(0); }

__device__ inline int64_t clamp_row(int64_t row, int64_t rows) { return row < rows ? row : rows - 1; }

// The adapters of a tile's rows, one after the other, and the rows that each has.
struct Adapters {
    int id;                            // of the lane's row; -1: none
    uint64_t left;                     // rows not yet visited
    // `v`: the lane's id, by load()
    static __device__ int load(const int32_t *ids, int64_t row0, int64_t rows) { return ids[clamp_row(row0 + (threadIdx.x & 63), rows)]; }
    __device__ Adapters(int v, int64_t row0, int64_t rows, int adapters, int count)
    {
        const int lane = threadIdx.x & 63;
        id = lane < count && row0 + lane < rows && v >= 0 && v < adapters ? v : -1;
        left = __ballot(id >= 0);
    }
    __device__ bool next(int &adapter, uint64_t &mine)
    {
        if (!left) return false;
        adapter = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        mine = __ballot(id == adapter);
        left &= ~mine;
        return true;
    }
};

// --------------------------------------------------------------------------
// first product
// --------------------------------------------------------------------------
// Matrix instructions of eight reduction elements a lane, operands of the weights' type.  Codes of 8 bits are exact in all of them.
template <typename TW> struct Operand { typedef typename Vec8<TW>::type type; };
template <typename TW, typename TX> __device__ inline typename Operand<TW>::type operand(typename Vec8<TX>::type v)
{
    if constexpr (std::is_same<TW, TX>::value) return v;
    else return __builtin_convertvector(widen(v), typename Operand<TW>::type);
}
__device__ inline v4f multiply(v8bf x, v8bf w, v4f acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, acc, 0, 0, 0); }
__device__ inline v4f multiply(v8h x, v8h w, v4f acc) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, acc, 0, 0, 0); }
__device__ inline v4f multiply(v8f x, v8f w, v4f acc)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], w[i], acc, 0, 0, 0);
    return acc;
}

// Eight elements from column `col` on, without a branch, so that several loads can be under way: columns beyond the last are
// read from it.
template <typename T, bool VEC> __device__ inline typename Vec8<T>::type columns8(const T *row, int64_t col, int64_t cols)
{
    typedef typename Vec8<T>::type V;
    if constexpr (VEC) return *(const V *)(row + min(col, cols - 8));
    else {
        union { V v; T e[8]; } u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.e[i] = row[min(col + i, cols - 1)];
        return u.v;
    }
}
// The same with 0 for the columns beyond: elements of a reduction.
template <typename T, bool VEC> __device__ inline typename Vec8<T>::type piece(const T *row, int64_t k, int64_t cols)
{
    typedef typename Vec8<T>::type V;
    union { V v; T e[8]; } u;
    u.v = columns8<T, VEC>(row, k, cols);
    if constexpr (VEC) return k < cols ? u.v : V(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) u.e[i] = k + i < cols ? u.e[i] : T(0);
    return u.v;
}

struct FirstArgs {
    const void *x, *w;
    int64_t stride, rows, K, chunk;    // chunk: reduction elements of a workgroup, a multiple of 64
    const float *step, *scale;
    const int32_t *ids;
    int R, adapters, slots;
    float *out;                        // [splits, rows, R]: a sum for each part of the reduction
};

// Column of half `half` of a lane's sixteen elements in a step of 64: four lanes read 64 bytes of a row in one instruction.
template <typename TX> __device__ inline int half_at(int q, int half) { return sizeof(TX) == 1 ? 16 * q + 8 * half : 32 * half + 8 * q; }

// A tile of 32 rows by 16 RT ranks, and a part of the reduction.  The four wavefronts take its steps of 64 elements in turn
// and add up in LDS.  Several steps' loads are issued before the first one's products: a wavefront waits for memory
// once per batch.
template <typename TX, typename TW, int RT, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_first(FirstArgs a)
{
    constexpr int kBatch = sizeof(TW) == 2 ? (RT == 1 ? 4 : 2) : (RT == 1 ? 2 : 1);
    typedef typename Vec8<TX>::type XV;
    typedef typename Vec8<TW>::type WV;
    __shared__ float sums[4][kRows][16 * RT];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    const int64_t row0 = (int64_t)(blockIdx.x / a.slots) * kRows;
    const int slot = blockIdx.x % a.slots, r0 = blockIdx.y * 16 * RT;
    const int64_t k0 = (int64_t)blockIdx.z * a.chunk, k1 = min(k0 + a.chunk, a.K);
    float *out = a.out + (int64_t)blockIdx.z * a.rows * a.R;
    const TX *xr[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) xr[m] = (const TX *)a.x + clamp_row(row0 + 16 * m + l, a.rows) * a.stride;

    Adapters of(Adapters::load(a.ids, row0, a.rows), row0, a.rows, a.adapters, kRows);
    if (slot == 0) {                                   // rows without an adapter
        const uint64_t none = ~of.left;
        for (int i = threadIdx.x; i < kRows * 16 * RT; i += 256) {
            const int row = i / (16 * RT), r = r0 + i % (16 * RT);
            if (((none >> row) & 1) && row0 + row < a.rows && r < a.R) out[(row0 + row) * a.R + r] = 0.0f;
        }
    }
    int adapter;
    uint64_t mine;
    for (int turn = 0; of.next(adapter, mine); ++turn) {
        if (turn % a.slots != slot) continue;
        const TW *wr[RT];
#pragma unroll
        for (int n = 0; n < RT; ++n) wr[n] = (const TW *)a.w + ((int64_t)adapter * a.R + min(r0 + 16 * n + l, a.R - 1)) * a.K;
        v4f acc[2][RT];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < RT; ++n) acc[m][n] = v4f(0);
        int64_t k = k0 + 64 * wave;
        if constexpr (VEC) {
            for (; k + 256 * (kBatch - 1) + 64 <= k1; k += 256 * kBatch) {
                XV x[kBatch][2][2];
                WV w[kBatch][2][RT];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int64_t c = k + 256 * b + half_at<TX>(q, half);
#pragma unroll
                        for (int m = 0; m < 2; ++m) x[b][half][m] = *(const XV *)(xr[m] + c);
#pragma unroll
                        for (int n = 0; n < RT; ++n) w[b][half][n] = *(const WV *)(wr[n] + c);
                    }
                loads_first();
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            const typename Operand<TW>::type xm = operand<TW, TX>(x[b][half][m]);
#pragma unroll
                            for (int n = 0; n < RT; ++n) acc[m][n] = multiply(xm, w[b][half][n], acc[m][n]);
                        }
            }
        }
        for (; k < k1; k += 256) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int64_t c = k + half_at<TX>(q, half);
                typename Operand<TW>::type x[2];
#pragma unroll
                for (int m = 0; m < 2; ++m) x[m] = operand<TW, TX>(piece<TX, VEC>(xr[m], c, k1));
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    const WV w = piece<TW, VEC>(wr[n], c, k1);
#pragma unroll
                    for (int m = 0; m < 2; ++m) acc[m][n] = multiply(x[m], w, acc[m][n]);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < RT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[wave][16 * m + 4 * q + i][16 * n + l] = acc[m][n][i];
        __syncthreads();
        const float scale = a.scale[adapter];
        for (int i = threadIdx.x; i < kRows * 16 * RT; i += 256) {
            const int row = i / (16 * RT), col = i % (16 * RT);
            if (!((mine >> row) & 1) || r0 + col >= a.R) continue;
            const float s = (sums[0][row][col] + sums[1][row][col]) + (sums[2][row][col] + sums[3][row][col]);
            out[(row0 + row) * a.R + r0 + col] = s * (a.step ? scale * a.step[row0 + row] : scale);
        }
    }
}

// --------------------------------------------------------------------------
// second product
// --------------------------------------------------------------------------
struct SecondArgs {
    const float *h;                    // [splits, rows, R]
    float *h_out;                      // [rows, R], the sum of the parts; NULL where there is one
    const void *w, *base;
    void *out;
    int64_t base_stride, out_stride, rows, C;
    const float *base_step;
    const int32_t *ids;
    int R, splits, adapters, out_type, column_tiles;
};

// A wavefront does 16 rows by 128 columns, with binary32 matrix instructions: H stays in binary32, and a lane's eight
// neighbouring columns are eight instructions, so neither W nor Y needs a transposition and both move in vectors.  The ranks
// come sixteen at a time, their products added to the row's sum where the row has the adapter.
constexpr int kSecondRows = 16;
__host__ __device__ inline int second_pitch(int R) { return (R + 15) / 16 * 16 + 1; }

template <typename T> __device__ inline void store_columns(void *data, int64_t at, int64_t col, int64_t cols, v8f v, bool vec)
{
    T *p = (T *)data + at + col;
    if (vec) {
        if (col < cols) store8(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) p[i] = (T)v[i];
    }
}

template <typename TW, typename TB, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_second(SecondArgs a)
{
    typedef typename Vec8<TW>::type WV;
    typedef typename Vec8<TB>::type BV;
    extern __shared__ float hs[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    const int64_t row0 = (int64_t)(blockIdx.x / a.column_tiles) * kSecondRows;
    const int tile = blockIdx.x % a.column_tiles, pitch = second_pitch(a.R);
    const int64_t col = ((int64_t)tile * (blockDim.x / 64) + wave) * 128 + 8 * l;

    const int id = Adapters::load(a.ids, row0, a.rows);
    BV base[4];
    if (a.base) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            base[i] = columns8<TB, VEC>((const TB *)a.base + clamp_row(row0 + 4 * q + i, a.rows) * a.base_stride, col, a.C);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) base[i] = BV(0);
    }
    float factor[4];                                   // without factors any number that can be read
    const float *from = a.base_step ? a.base_step : a.h;
#pragma unroll
    for (int i = 0; i < 4; ++i) factor[i] = from[a.base_step ? clamp_row(row0 + 4 * q + i, a.rows) : 0];
    loads_first();
    Adapters of(id, row0, a.rows, a.adapters, kSecondRows);
    // the ranks r0 to r0 + 15 of one adapter's W, those beyond R 0
    auto ranks = [&](int adapter, int r0, WV (&v)[4]) {
#pragma unroll
        for (int s = 0; s < 4; ++s)
            v[s] = columns8<TW, VEC>((const TW *)a.w + ((int64_t)adapter * a.R + min(r0 + 4 * s + q, a.R - 1)) * a.C, col, a.C);
#pragma unroll
        for (int s = 0; s < 4; ++s) v[s] = r0 + 4 * s + q < a.R ? v[s] : WV(0);
    };
    int adapter = 0;
    uint64_t mine = 0;
    bool more = of.next(adapter, mine);
    WV w[4];
    ranks(adapter, 0, w);

    for (int row = threadIdx.x >> 4; row < kSecondRows; row += blockDim.x >> 4)
        for (int r = l; r < pitch - 1; r += 16) {
            const int64_t at = clamp_row(row0 + row, a.rows) * a.R + min(r, a.R - 1);
            float s = 0.0f;
            for (int p = 0; p < a.splits; p += 4) {
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = a.h[min(p + j, a.splits - 1) * a.rows * a.R + at];
                loads_first();
#pragma unroll
                for (int j = 0; j < 4; ++j) s += p + j < a.splits ? v[j] : 0.0f;
            }
            if (r >= a.R) s = 0.0f;
            else if (tile == 0 && a.h_out && row0 + row < a.rows) a.h_out[at] = s;
            hs[row * pitch + r] = s;
        }
    __syncthreads();
    v8f acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = widen(base[i]);
    if (a.base_step) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= factor[i];
    }
    int r0 = 0;
    while (more) {
        v8f wv[4];
        float h[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            wv[s] = widen(w[s]);
            h[s] = hs[l * pitch + r0 + 4 * s + q];
        }
        const uint64_t rows = mine;
        r0 += 16;
        if (r0 >= a.R) {
            r0 = 0;
            more = of.next(adapter, mine);
        }
        if (more) ranks(adapter, r0, w);
        v4f y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = v4f(0);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(h[s], wv[s][j], y[j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool own = (rows >> (4 * q + i)) & 1;
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[i][j] += own ? y[j][i] : 0.0f;
        }
    }
    if (a.out_type == PWLQ_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (row0 + 4 * q + i < a.rows) store_columns<float>(a.out, (row0 + 4 * q + i) * a.out_stride, col, a.C, acc[i], VEC);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (row0 + 4 * q + i < a.rows) store_columns<TW>(a.out, (row0 + 4 * q + i) * a.out_stride, col, a.C, acc[i], VEC);
    }
}

// --------------------------------------------------------------------------
// both products for few rows
// --------------------------------------------------------------------------
// One rank of one row.
template <typename TX, typename TW, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_first_token(FirstArgs a)
{
    __shared__ float slots[16];
    const int64_t row = blockIdx.y;
    const int r = blockIdx.x, id = a.ids[row];
    float s = 0.0f;
    if (id >= 0 && id < a.adapters) {
        const TX *x = (const TX *)a.x + row * a.stride;
        const TW *w = (const TW *)a.w + ((int64_t)id * a.R + r) * a.K;
        v8f t = v8f(0);
#pragma unroll 2
        for (int64_t k = 8 * threadIdx.x; k < a.K; k += 8 * 256) t += widen(piece<TX, VEC>(x, k, a.K)) * widen(piece<TW, VEC>(w, k, a.K));
        s = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
        s = block_sum(s, slots, 256) * (a.step ? a.scale[id] * a.step[row] : a.scale[id]);
    }
    if (threadIdx.x == 0) a.out[row * a.R + r] = s;
}

// 512 columns of one row; the four wavefronts share the ranks.
template <typename TW, typename TB, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_second_token(SecondArgs a)
{
    __shared__ v8f sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.y, col = (int64_t)blockIdx.x * 512 + 8 * lane;
    const int id = a.ids[row];
    v8f y = v8f(0), base = v8f(0);
    if (a.base && wave == 0) base = widen(piece<TB, VEC>((const TB *)a.base + row * a.base_stride, col, a.C));
    if (id >= 0 && id < a.adapters) {
        const TW *w = (const TW *)a.w + (int64_t)id * a.R * a.C;
#pragma unroll 4
        for (int r = wave; r < a.R; r += 4) y += a.h[row * a.R + r] * widen(piece<TW, VEC>(w + (int64_t)r * a.C, col, a.C));
    }
    sums[wave][lane] = y;
    __syncthreads();
    if (wave) return;
    y = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    y += a.base_step ? base * a.base_step[row] : base;
    if (a.out_type == PWLQ_F32) store_columns<float>(a.out, row * a.out_stride, col, a.C, y, VEC);
    else store_columns<TW>(a.out, row * a.out_stride, col, a.C, y, VEC);
}

// Both products of one row in one launch, for 512 columns: the row's H is computed by each of its workgroups anew, which costs
// reading down again from L2 but no second launch and no wait for it.  The sixteen wavefronts share the ranks of both products.
struct TokenArgs {
    const void *x, *down, *up, *base;
    void *out;
    int64_t x_stride, base_stride, out_stride, K, C;
    const float *x_step, *base_step, *scale;
    const int32_t *ids;
    float *h;
    int R, adapters, base_type, out_type;
};
constexpr int kTokenThreads = 1024, kTokenColumns = 512, kTokenWaves = kTokenThreads / 64, kTokenRanks = 64;

template <typename TX, typename TW, bool VEC>
__global__ __launch_bounds__(kTokenThreads) void k_adapter_token(TokenArgs a)
{
    typedef typename Vec8<TX>::type XV;
    typedef typename Vec8<TW>::type WV;
    constexpr int kAhead = sizeof(TW) == 2 ? 8 : 4;            // vectors of a lane in flight
    __shared__ float hs[kTokenRanks];
    __shared__ v8f sums[kTokenWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.y, col0 = (int64_t)blockIdx.x * kTokenColumns, col = col0 + 8 * lane;
    const int id = a.ids[row];
    float base = 0.0f;
    if (a.base && threadIdx.x < kTokenColumns && col0 + threadIdx.x < a.C) {
        const int64_t at = row * a.base_stride + col0 + threadIdx.x;
        base = (a.base_type == PWLQ_F32 ? ((const float *)a.base)[at] : widen(((const TW *)a.base)[at])) * (a.base_step ? a.base_step[row] : 1.0f);
    }
    v8f y = v8f(0);
    if (id >= 0 && id < a.adapters) {
        const TW *up = (const TW *)a.up + (int64_t)id * a.R * a.C;
        const WV ahead = piece<TW, VEC>(up + (int64_t)min(wave, a.R - 1) * a.C, col, a.C);
        const TX *x = (const TX *)a.x + row * a.x_stride;
        const float scale = a.x_step ? a.scale[id] * a.x_step[row] : a.scale[id];
        for (int r = wave; r < a.R; r += kTokenWaves) {
            const TW *w = (const TW *)a.down + ((int64_t)id * a.R + r) * a.K;
            v8f t = v8f(0);
            int64_t k = 0;
            if constexpr (VEC) {
                // vectors beyond the row are read from its last one and count nothing
                for (; k < a.K; k += 512 * kAhead) {
                    XV xv[kAhead];
                    WV wv[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int64_t c = min(k + 512 * i + 8 * lane, a.K - 8);
                        xv[i] = *(const XV *)(x + c);
                        wv[i] = *(const WV *)(w + c);
                    }
                    loads_first();
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const v8f p = widen(xv[i]) * widen(wv[i]);
                        t += k + 512 * i + 8 * lane < a.K ? p : v8f(0);
                    }
                }
            } else {
                for (k = 8 * lane; k < a.K; k += 512) t += widen(piece<TX, VEC>(x, k, a.K)) * widen(piece<TW, VEC>(w, k, a.K));
            }
            const float s = wave_sum(((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7])));
            if (lane == 0) hs[r] = s * scale;
        }
        __syncthreads();
        if (blockIdx.x == 0 && threadIdx.x < a.R) a.h[row * a.R + threadIdx.x] = hs[threadIdx.x];
        if (wave < a.R) y = hs[wave] * widen(ahead);
        for (int r = wave + kTokenWaves; r < a.R; r += kTokenWaves) y += hs[r] * widen(piece<TW, VEC>(up + (int64_t)r * a.C, col, a.C));
    } else if (blockIdx.x == 0 && threadIdx.x < a.R) {
        a.h[row * a.R + threadIdx.x] = 0.0f;
    }
    sums[wave][lane] = y;
    __syncthreads();
    if (threadIdx.x >= kTokenColumns || col0 + threadIdx.x >= a.C) return;
    float s = 0.0f;
#pragma unroll
    for (int g = 0; g < kTokenWaves; ++g) s += ((const float *)sums[g])[threadIdx.x];
    const int64_t at = row * a.out_stride + col0 + threadIdx.x;
    if (a.out_type == PWLQ_F32) ((float *)a.out)[at] = base + s;
    else ((TW *)a.out)[at] = (TW)(base + s);
}

// --------------------------------------------------------------------------
// outer products
// --------------------------------------------------------------------------
struct OuterArgs {
    const float *h;                    // [rows, R]
    const void *x;
    int64_t stride, rows, C, span;     // span: rows of a workgroup, a multiple of 64
    const float *step;
    const int32_t *ids;
    int R, adapters, column_tiles, splits;
    float *out;                        // [splits, adapters, R, C]
    int32_t *present;                  // [splits, adapters]: whether the part has rows of the adapter; NULL where there is one part
};

// 16 RT ranks by 128 columns of one adapter's gradient, over a part of the rows.  The rows of the adapter are listed in LDS
// first, 512 at a time, so that no other row is read.  As in the second product a lane's eight neighbouring columns are eight
// binary32 matrix instructions; a step is four rows, and a wavefront has several steps' loads in flight.
constexpr int kListed = 512;

template <typename TX, int RT, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_outer(OuterArgs a)
{
    constexpr int kSteps = RT == 4 ? 4 : 8;
    __shared__ v4f sums[2][RT * 8][64];
    __shared__ int list[kListed];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    const int64_t col = (int64_t)(blockIdx.x % a.column_tiles) * 128 + 8 * l;
    const int r0 = blockIdx.x / a.column_tiles * 16 * RT, adapter = blockIdx.y, split = blockIdx.z;
    const int64_t t0 = split * a.span, t1 = min(t0 + a.span, a.rows);
    v4f acc[RT][8];
#pragma unroll
    for (int n = 0; n < RT; ++n)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[n][j] = v4f(0);
    bool any = false;
    for (int64_t t = t0; t < t1; t += kListed) {
        int id[kListed / 64];
#pragma unroll
        for (int g = 0; g < kListed / 64; ++g) id[g] = a.ids[clamp_row(t + 64 * g + lane, t1)];
        loads_first();
        int count = 0;
        __syncthreads();
#pragma unroll
        for (int g = 0; g < kListed / 64; ++g) {
            const uint64_t mine = __ballot(id[g] == adapter && t + 64 * g + lane < t1);
            if (g % 4 == wave && ((mine >> lane) & 1)) list[count + __builtin_popcountll(mine & ((1ull << lane) - 1))] = 64 * g + lane;
            count += __builtin_popcountll(mine);
        }
        __syncthreads();
        any |= count != 0;
        for (int first = 4 * kSteps * wave; first < count; first += 16 * kSteps) {
            typename Vec8<TX>::type x[kSteps];
            float h[kSteps][RT], step[kSteps];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int64_t row = t + list[min(first + 4 * s + q, count - 1)];
                x[s] = columns8<TX, VEC>((const TX *)a.x + row * a.stride, col, a.C);
#pragma unroll
                for (int n = 0; n < RT; ++n) h[s][n] = a.h[row * a.R + min(r0 + 16 * n + l, a.R - 1)];
                if constexpr (sizeof(TX) == 1) step[s] = a.step[row];
            }
            loads_first();
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const bool own = first + 4 * s + q < count;
                v8f xv = widen(x[s]);
                if (!own) xv = v8f(0);
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    float hv = h[s][n];
                    if constexpr (sizeof(TX) == 1) hv *= step[s];
                    hv = own ? hv : 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(hv, xv[j], acc[n][j], 0, 0, 0);
                }
            }
        }
    }
    if (a.present) {
        if (blockIdx.x == 0 && threadIdx.x == 0) a.present[split * a.adapters + adapter] = any;
        if (!any) return;
    }
    if (wave >= 2) {
#pragma unroll
        for (int n = 0; n < RT; ++n)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[wave - 2][8 * n + j][lane] = acc[n][j];
    }
    __syncthreads();
    if (wave < 2) {
#pragma unroll
        for (int n = 0; n < RT; ++n)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[n][j] += sums[wave][8 * n + j][lane];
    }
    __syncthreads();
    if (wave == 1) {
#pragma unroll
        for (int n = 0; n < RT; ++n)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[0][8 * n + j][lane] = acc[n][j];
    }
    __syncthreads();
    if (wave) return;
    float *out = a.out + ((int64_t)split * a.adapters + adapter) * a.R * a.C;
#pragma unroll
    for (int n = 0; n < RT; ++n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[n][j] += sums[0][8 * n + j][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 16 * n + 4 * q + i;
            v8f v;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = acc[n][j][i];
            if (r < a.R) store_columns<float>(out, (int64_t)r * a.C, col, a.C, v, VEC);
        }
    }
}

// Parts of one or two gradients added up in order.
struct JoinArgs {
    const float *part[2];
    const int32_t *present[2];
    float *out[2];
    int64_t each[2];                   // R C
    int splits[2];
    int adapters;
};
__global__ __launch_bounds__(256) void k_adapter_join(JoinArgs a)
{
    const int which = blockIdx.z, adapter = blockIdx.y, lane = threadIdx.x & 63;
    const int64_t each = a.each[which], n = each * a.adapters;
    const float *part = a.part[which] + adapter * each;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i - lane < each; i += (int64_t)gridDim.x * 256) {
        const int64_t at = min(i, each - 1);
        float s = 0.0f;
        for (int p0 = 0; p0 < a.splits[which]; p0 += 64) {
            uint64_t parts = __ballot(p0 + lane < a.splits[which] && a.present[which][(p0 + lane) * a.adapters + adapter]);
            while (parts) {                              // four loads at a time
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = parts ? part[(p0 + __builtin_ctzll(parts)) * n + at] : 0.0f;
                    parts &= parts - 1;
                }
                loads_first();
                s += (v[0] + v[1]) + (v[2] + v[3]);
            }
        }
        if (i < each) a.out[which][adapter * each + i] = s;
    }
}

__global__ void k_zero(float *a, int64_t na, float *b, int64_t nb)
{
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t j = i; j < na; j += step) a[j] = 0.0f;
    for (int64_t j = i; j < nb; j += step) b[j] = 0.0f;
}

// --------------------------------------------------------------------------
// launches
// --------------------------------------------------------------------------
constexpr int64_t kTokenRows = 16;     // up to so many rows each is done by itself

int rank_tiles(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : 4; }
int rank_blocks(int R) { return (R + 16 * rank_tiles(R) - 1) / (16 * rank_tiles(R)); }

// Parts of the first product's reduction: workgroups for the whole chip, with two steps for each wavefront at least.
int first_splits(int64_t T, int64_t K, int R)
{
    if (T <= kTokenRows) return 1;
    const int64_t wgs = (T + kRows - 1) / kRows * rank_blocks(R);
    return (int)std::max<int64_t>(1, std::min<int64_t>((640 + wgs - 1) / wgs, (K + 511) / 512));
}
int64_t first_chunk(int64_t K, int splits) { return ((K + splits - 1) / splits + 63) / 64 * 64; }

// Parts of the rows for an outer product.
int64_t outer_span(int64_t T, int64_t C, int R)
{
    const int64_t wgs = (C + 127) / 128 * rank_blocks(R), most = rank_tiles(R) == 4 ? 256 : 640;
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>((most + wgs - 1) / wgs, (T + 63) / 64));
    return ((T + splits - 1) / splits + 63) / 64 * 64;
}
int outer_splits(int64_t T, int64_t C, int R) { return (int)((T + outer_span(T, C, R) - 1) / outer_span(T, C, R)); }

struct Carver {                        // offsets of a workspace's parts, 256-byte aligned
    char *base;
    size_t at = 0;
    template <typename T> T *take(int64_t n)
    {
        T *p = base ? (T *)(base + at) : nullptr;
        at += ((size_t)n * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

struct BackwardSpace {
    float *dh, *parts, *down, *up;
    int32_t *has_down, *has_up;
    size_t bytes;
    BackwardSpace(void *workspace, int64_t T, int64_t K, int64_t N, int R, int adapters)
    {
        Carver c = {(char *)workspace};
        const int splits = first_splits(T, N, R), sd = outer_splits(T, K, R), su = outer_splits(T, N, R);
        dh = c.take<float>(T * R);
        parts = splits > 1 ? c.take<float>(splits * T * R) : dh;
        down = sd > 1 ? c.take<float>((int64_t)sd * adapters * R * K) : nullptr;
        up = su > 1 ? c.take<float>((int64_t)su * adapters * R * N) : nullptr;
        has_down = c.take<int32_t>((int64_t)sd * adapters);
        has_up = c.take<int32_t>((int64_t)su * adapters);
        bytes = c.at;
    }
};

template <typename TX, typename TW> void first_as(FirstArgs a, bool vec, hipStream_t stream)
{
    if (a.rows <= kTokenRows) {
        const dim3 grid(a.R, (unsigned)a.rows);
        if (vec) k_adapter_first_token<TX, TW, true><<<grid, 256, 0, stream>>>(a);
        else k_adapter_first_token<TX, TW, false><<<grid, 256, 0, stream>>>(a);
        return;
    }
    const int64_t tiles = (a.rows + kRows - 1) / kRows, splits = (a.K + a.chunk - 1) / a.chunk;
    a.slots = (int)std::min<int64_t>(std::min(a.adapters, kRows), std::max<int64_t>(1, 2048 / (tiles * splits * rank_blocks(a.R))));
    const dim3 grid((unsigned)(tiles * a.slots), rank_blocks(a.R), (unsigned)splits);
#define PWLQ_FIRST(RT)                                                                          \
    do {                                                                                        \
        if (vec) k_adapter_first<TX, TW, RT, true><<<grid, 256, 0, stream>>>(a);                \
        else k_adapter_first<TX, TW, RT, false><<<grid, 256, 0, stream>>>(a);                   \
    } while (0)
    if (rank_tiles(a.R) == 1) PWLQ_FIRST(1);
    else if (rank_tiles(a.R) == 2) PWLQ_FIRST(2);
    else PWLQ_FIRST(4);
#undef PWLQ_FIRST
}

void first(const FirstArgs &a, int x_type, int w_type, bool vec, hipStream_t stream)
{
    if (w_type == PWLQ_F32) x_type == PWLQ_I8 ? first_as<int8_t, float>(a, vec, stream) : first_as<float, float>(a, vec, stream);
    else if (w_type == PWLQ_BF16) x_type == PWLQ_I8 ? first_as<int8_t, bf16>(a, vec, stream) : first_as<bf16, bf16>(a, vec, stream);
    else x_type == PWLQ_I8 ? first_as<int8_t, f16>(a, vec, stream) : first_as<f16, f16>(a, vec, stream);
}

template <typename TW, typename TB> void second_as(SecondArgs a, bool vec, hipStream_t stream)
{
    if (a.rows <= kTokenRows && a.splits == 1) {
        const dim3 grid((unsigned)((a.C + 511) / 512), (unsigned)a.rows);
        if (vec) k_adapter_second_token<TW, TB, true><<<grid, 256, 0, stream>>>(a);
        else k_adapter_second_token<TW, TB, false><<<grid, 256, 0, stream>>>(a);
        return;
    }
    const int64_t tiles = (a.rows + kSecondRows - 1) / kSecondRows, columns = (a.C + 127) / 128;
    const int waves = tiles * columns < 2048 ? 1 : 4;
    a.column_tiles = (int)((columns + waves - 1) / waves);
    const size_t lds = sizeof(float) * kSecondRows * second_pitch(a.R);
    const unsigned grid = (unsigned)(tiles * a.column_tiles);
    if (vec) k_adapter_second<TW, TB, true><<<grid, 64 * waves, lds, stream>>>(a);
    else k_adapter_second<TW, TB, false><<<grid, 64 * waves, lds, stream>>>(a);
}

void second(const SecondArgs &a, int w_type, int base_type, bool vec, hipStream_t stream)
{
    if (w_type == PWLQ_F32) second_as<float, float>(a, vec, stream);
    else if (w_type == PWLQ_BF16) base_type == PWLQ_F32 ? second_as<bf16, float>(a, vec, stream) : second_as<bf16, bf16>(a, vec, stream);
    else base_type == PWLQ_F32 ? second_as<f16, float>(a, vec, stream) : second_as<f16, f16>(a, vec, stream);
}

template <typename TX> void outer_as(const OuterArgs &a, bool vec, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.column_tiles * rank_blocks(a.R)), a.adapters, a.splits);
#define PWLQ_OUTER(RT)                                                                          \
    do {                                                                                        \
        if (vec) k_adapter_outer<TX, RT, true><<<grid, 256, 0, stream>>>(a);                    \
        else k_adapter_outer<TX, RT, false><<<grid, 256, 0, stream>>>(a);                       \
    } while (0)
    if (rank_tiles(a.R) == 1) PWLQ_OUTER(1);
    else if (rank_tiles(a.R) == 2) PWLQ_OUTER(2);
    else PWLQ_OUTER(4);
#undef PWLQ_OUTER
}

void outer(const pwlq_rows &x, int64_t T, int64_t C, int R, int adapters, const float *h, const int32_t *ids, float *out, float *parts,
           int32_t *present, hipStream_t stream)
{
    OuterArgs a = {};
    a.h = h;
    a.x = x.data;
    a.stride = x.stride;
    a.rows = T;
    a.C = C;
    a.span = outer_span(T, C, R);
    a.splits = outer_splits(T, C, R);
    a.step = x.step;
    a.ids = ids;
    a.R = R;
    a.adapters = adapters;
    a.column_tiles = (int)((C + 127) / 128);
    a.out = a.splits > 1 ? parts : out;
    a.present = a.splits > 1 ? present : nullptr;
    const bool vec = C % 8 == 0 && vectors(x, T) && aligned16(a.out);
    if (x.type == PWLQ_F32) outer_as<float>(a, vec, stream);
    else if (x.type == PWLQ_BF16) outer_as<bf16>(a, vec, stream);
    else if (x.type == PWLQ_F16) outer_as<f16>(a, vec, stream);
    else outer_as<int8_t>(a, vec, stream);
}

bool whole_vectors(int64_t C, const void *w) { return C % 8 == 0 && aligned16(w); }

// Whether few rows go through one launch.
bool by_token(const pwlq_adapter_args &a)
{
    return a.T <= kTokenRows && a.R <= kTokenRanks;
}

template <typename TX, typename TW> void token_as(const TokenArgs &a, int64_t rows, bool vec, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.C + kTokenColumns - 1) / kTokenColumns), (unsigned)rows);
    if (vec) k_adapter_token<TX, TW, true><<<grid, kTokenThreads, 0, stream>>>(a);
    else k_adapter_token<TX, TW, false><<<grid, kTokenThreads, 0, stream>>>(a);
}

void token(const pwlq_adapter_args &a, hipStream_t stream)
{
    TokenArgs t = {};
    t.x = a.x.data;
    t.down = a.down;
    t.up = a.up;
    t.base = a.base.data;
    t.out = a.out.data;
    t.x_stride = a.x.stride;
    t.base_stride = a.base.stride;
    t.out_stride = a.out.stride;
    t.K = a.K;
    t.C = a.N;
    t.x_step = a.x.step;
    t.base_step = a.base.data ? a.base.step : nullptr;
    t.scale = a.scale;
    t.ids = a.ids;
    t.h = a.h;
    t.R = a.R;
    t.adapters = a.adapters;
    t.base_type = a.base.type;
    t.out_type = a.out.type;
    const bool vec = whole_vectors(a.K, a.down) && whole_vectors(a.N, a.up) && vectors(a.x, a.T), packed = a.x.type == PWLQ_I8;
    if (a.weight_type == PWLQ_F32) packed ? token_as<int8_t, float>(t, a.T, vec, stream) : token_as<float, float>(t, a.T, vec, stream);
    else if (a.weight_type == PWLQ_BF16) packed ? token_as<int8_t, bf16>(t, a.T, vec, stream) : token_as<bf16, bf16>(t, a.T, vec, stream);
    else packed ? token_as<int8_t, f16>(t, a.T, vec, stream) : token_as<f16, f16>(t, a.T, vec, stream);
}

} // namespace

size_t adapter_workspace(int64_t T, int64_t K, int R)
{
    const int splits = first_splits(T, K, R);
    return splits > 1 ? (size_t)splits * (size_t)T * (size_t)R * sizeof(float) : 0;
}

void adapter_forward(const pwlq_adapter_args &a, void *workspace, hipStream_t stream)
{
    if (by_token(a)) {
        token(a, stream);
        return;
    }
    FirstArgs f = {};
    f.x = a.x.data;
    f.w = a.down;
    f.stride = a.x.stride;
    f.rows = a.T;
    f.K = a.K;
    const int splits = first_splits(a.T, a.K, a.R);
    f.chunk = first_chunk(a.K, splits);
    f.step = a.x.step;
    f.scale = a.scale;
    f.ids = a.ids;
    f.R = a.R;
    f.adapters = a.adapters;
    const int parts = (int)((a.K + f.chunk - 1) / f.chunk);
    f.out = parts > 1 ? (float *)workspace : a.h;
    first(f, a.x.type, a.weight_type, whole_vectors(a.K, a.down) && vectors(a.x, a.T), stream);
    SecondArgs s = {};
    s.h = f.out;
    s.h_out = parts > 1 ? a.h : nullptr;
    s.w = a.up;
    s.base = a.base.data;
    s.out = a.out.data;
    s.base_stride = a.base.stride;
    s.out_stride = a.out.stride;
    s.rows = a.T;
    s.C = a.N;
    s.base_step = a.base.data ? a.base.step : nullptr;
    s.ids = a.ids;
    s.R = a.R;
    s.splits = parts;
    s.adapters = a.adapters;
    s.out_type = a.out.type;
    second(s, a.weight_type, a.base.data ? a.base.type : PWLQ_F32, whole_vectors(a.N, a.up) && vectors(a.base, a.T) && vectors(a.out, a.T), stream);
}

size_t adapter_backward_workspace(int64_t T, int64_t K, int64_t N, int R, int adapters)
{
    return T ? BackwardSpace(nullptr, T, K, N, R, adapters).bytes : 0;
}

void adapter_backward(const pwlq_adapter_backward_args &a, void *workspace, hipStream_t stream)
{
    if (a.T == 0) {
        k_zero<<<256, 256, 0, stream>>>(a.d_down, (int64_t)a.adapters * a.R * a.K, a.d_up, (int64_t)a.adapters * a.R * a.N);
        return;
    }
    const BackwardSpace space(workspace, a.T, a.K, a.N, a.R, a.adapters);
    FirstArgs f = {};
    f.x = a.dy.data;
    f.w = a.up;
    f.stride = a.dy.stride;
    f.rows = a.T;
    f.K = a.N;
    f.chunk = first_chunk(a.N, first_splits(a.T, a.N, a.R));
    f.scale = a.scale;
    f.ids = a.ids;
    f.R = a.R;
    f.adapters = a.adapters;
    const int parts = (int)((a.N + f.chunk - 1) / f.chunk);
    f.out = parts > 1 ? space.parts : space.dh;
    first(f, a.dy.type, a.weight_type, whole_vectors(a.N, a.up) && vectors(a.dy, a.T), stream);
    SecondArgs s = {};
    s.h = f.out;
    s.h_out = parts > 1 ? space.dh : nullptr;
    s.w = a.down;
    s.base = a.dx_base.data;
    s.out = a.dx.data;
    s.base_stride = a.dx_base.stride;
    s.out_stride = a.dx.stride;
    s.rows = a.T;
    s.C = a.K;
    s.ids = a.ids;
    s.R = a.R;
    s.splits = parts;
    s.adapters = a.adapters;
    s.out_type = a.dx.type;
    second(s, a.weight_type, a.dx_base.data ? a.dx_base.type : PWLQ_F32,
           whole_vectors(a.K, a.down) && vectors(a.dx_base, a.T) && vectors(a.dx, a.T), stream);
    outer(a.x, a.T, a.K, a.R, a.adapters, space.dh, a.ids, a.d_down, space.down, space.has_down, stream);
    outer(a.dy, a.T, a.N, a.R, a.adapters, a.h, a.ids, a.d_up, space.up, space.has_up, stream);
    JoinArgs j = {};
    int n = 0;
    auto join = [&](const float *part, const int32_t *present, float *out, int64_t C) {
        const int splits = outer_splits(a.T, C, a.R);
        if (splits == 1) return;
        j.part[n] = part;
        j.present[n] = present;
        j.out[n] = out;
        j.each[n] = a.R * C;
        j.splits[n++] = splits;
    };
    join(space.down, space.has_down, a.d_down, a.K);
    join(space.up, space.has_up, a.d_up, a.N);
    j.adapters = a.adapters;
    if (n) {
        const int64_t most = std::max(j.each[0], j.each[1]);
        const dim3 grid((unsigned)std::min<int64_t>((most + 255) / 256, 1 << 16), a.adapters, n);
        k_adapter_join<<<grid, 256, 0, stream>>>(j);
    }
}

} // namespace pwlq_block
