// Low-rank adapters of many requests beside a shared projection, and their gradients.  Three products carry both directions,
// for matrices W [adapters, R, C] with the rank before the columns, and the rows t of a batch with adapter a(t):
//   first   H[t] = scale[a] X[t] W[a]^T             (forward: x, down; backward: dy, up)
//   second  Y[t] = base[t] + H[t] W[a]              (forward: h, up; backward: dh, down)
//   outer   G[a] = sum over its rows of H[t] (x) X[t]       (d_down: dh, x; d_up: h, dy)
// With ranks of 16 to 64 all three are bound by memory: per element of X or Y they do 2 R operations.
//
// Rows of one request are next to each other, so most tiles of rows have one adapter; a tile of several is done once for
// each, or rows of one adapter are collected into tiles: any order of ids is right, and a row's result does not depend on the others.
#include <algorithm>

#include "launch.h"
#include "rows.h"

#pragma clang fp contract(fast)

namespace pwlq_block {
namespace {

constexpr int kRows = 32;              // rows of a tile of the first product: two of the matrix instructions'

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

// SPAN neighbouring rows in tiles of at most ROWS rows of one adapter: the span's adapters in turn, the rows of each in order.
// Rows of one request are next to each other, so with a span of one tile most tiles have one adapter, and one of several is done
// once for each.  Where requests may alternate (a batch that decodes), a span of 256 rows collects full tiles of rows that need the
// same weights.  Rows without an adapter are adapter -1.
constexpr int kCollected = 256;
template <int ROWS, int SPAN> struct Tiles {
    static constexpr int kNone = 0x7fffffff, kGroups = SPAN < 64 ? 1 : SPAN / 64;
    int id[kGroups];                   // of the rows 64 g + lane; kNone beyond the last row
    uint64_t mine[kGroups];            // the rows of `adapter`
    int adapter, count, first, end;    // `count` of them, in the tiles [first, end)

    __device__ void load(const int32_t *ids, int64_t row0, int64_t rows)
    {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) id[g] = ids[clamp_row(row0 + 64 * g + (threadIdx.x & 63), rows)];
    }
    // `after`: adapters up to it are left out
    __device__ void start(int64_t row0, int64_t rows, int adapters, int after)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
            id[g] = 64 * g + lane >= SPAN || row0 + 64 * g + lane >= rows ? kNone : id[g] >= 0 && id[g] < adapters ? id[g] : -1;
        adapter = after;
        count = first = end = 0;
    }
    // Goes on to the adapter that has the tile; false: there are fewer tiles.
    __device__ bool seek(int tile)
    {
        while (tile >= end) {
            uint32_t left = 0;         // kNone less the next adapter
#pragma unroll
            for (int g = 0; g < kGroups; ++g)
                if (id[g] > adapter) left = max(left, (uint32_t)kNone - (uint32_t)id[g]);
            left = wave_max(left);
            if (left == 0) return false;
            adapter = (int)((uint32_t)kNone - left);
            count = 0;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                mine[g] = __ballot(id[g] == adapter);
                count += __builtin_popcountll(mine[g]);
            }
            first = end;
            end += (count + ROWS - 1) / ROWS;
        }
        return true;
    }
    __device__ int size(int tile) const { return min(ROWS, count - (tile - first) * ROWS); }
    // The tile's rows into `list`, by the wavefronts together.
    __device__ void rows(int tile, int *list, int waves) const
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        int before = -(tile - first) * ROWS;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int at = before + __builtin_popcountll(mine[g] & ((1ull << lane) - 1));
            if (g % waves == wave && ((mine[g] >> lane) & 1) && at >= 0 && at < ROWS) list[at] = 64 * g + lane;
            before += __builtin_popcountll(mine[g]);
        }
    }
};

// --------------------------------------------------------------------------
// first product
// --------------------------------------------------------------------------
// Matrix instructions of eight reduction elements a lane, operands of the weights' type.  Codes of 8 bits are exact in all of them.
// Products of binary16 values below its normal range (2^-14) are summed with an error of up to 2^-37 by measurement, which is
// 2^-13 of what one unit of such a value adds.
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

// Eight elements from column `col` on.  A vector that would reach past the row's end is the row's last eight instead, shifted by
// beyond(): in place of a branch, so that several loads can be under way, and nothing past the end is read.  Rows shorter than a
// vector go element by element (VEC false).
__device__ inline int64_t start_of(int64_t col, int64_t cols) { return min(col, cols - 8); }
__device__ inline int beyond(int64_t col, int64_t cols) { return (int)min(col - start_of(col, cols), (int64_t)8); }
template <typename T, bool VEC> __device__ inline typename Vec8<T>::type columns8(const T *row, int64_t col, int64_t cols)
{
    if constexpr (VEC) return load8(row + start_of(col, cols));
    else {
        union { typename Vec8<T>::type v; T e[8]; } u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.e[i] = row[min(col + i, cols - 1)];
        return u.v;
    }
}
// Of such a vector the elements of a reduction: those from `col` on and before `end` (which ends the row or a run of vectors), 0
// for the others, each element once in all.
template <typename T, bool VEC> __device__ inline typename Vec8<T>::type only(typename Vec8<T>::type v, int64_t col, int64_t end, int64_t cols)
{
    union { typename Vec8<T>::type v; T e[8]; } u;
    u.v = v;
    const int skip = VEC ? (col < end ? beyond(col, cols) : 8) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) u.e[i] = VEC ? (i >= skip ? u.e[i] : T(0)) : (col + i < end ? u.e[i] : T(0));
    return u.v;
}

// A vector of a row that begins between two dwords, as the dwords that hold it, and cut out of them: as vectors of their own, 2070 rows
// of 4097 columns of bfloat16 take 21.6 us, so 10.0 (of 4096 8.7).  `row` is the dword that the row begins in and `shift` where in it.
// The dword behind is one that holds the vector's last bytes, or, where there are none in it, the one before.
template <typename T, bool ODD> struct Loaded {
    typename Vec8<T>::type v;
    __device__ void load(const T *row, int, int64_t col) { v = load8(row + col); }
    __device__ typename Vec8<T>::type get(int) const { return v; }
};
template <typename T> struct Loaded<T, true> {
    static constexpr int kWords = 8 * sizeof(T) / 4;
    typedef uint32_t words __attribute__((ext_vector_type(kWords), aligned(4)));
    words v;
    uint32_t end;
    __device__ void load(const T *row, int shift, int64_t col)
    {
        const uint32_t *p = (const uint32_t *)(row + col);
        v = *(const words *)p;
        end = p[shift ? kWords : kWords - 1];
    }
    __device__ typename Vec8<T>::type get(int shift) const
    {
        union { uint32_t w[kWords]; typename Vec8<T>::type v; } u;
#pragma unroll
        for (int i = 0; i < kWords; ++i) u.w[i] = __builtin_amdgcn_alignbyte(i + 1 < kWords ? v[i + 1] : end, v[i], shift);
        return u.v;
    }
};
template <typename T, bool ODD> __device__ inline int shift_of(const T *row) { return ODD && sizeof(T) < 4 ? (int)((uintptr_t)row & 3) : 0; }
template <typename T> __device__ inline const T *dword_of(const T *row, int shift) { return (const T *)((const char *)row - shift); }

struct FirstArgs {
    const void *x, *w;
    int64_t stride, rows, K, chunk;    // chunk: reduction elements of a workgroup, a multiple of 64
    const float *step, *scale;
    const int32_t *ids;
    int R, adapters, turns;            // turns: workgroups that share a span's tiles
    float *out;                        // [splits, rows, R]: a sum for each part of the reduction
};

// Column of half `half` of a lane's sixteen elements in a step of 64: four lanes read 64 bytes of a row in one instruction.
template <typename TX> __device__ inline int half_at(int q, int half) { return sizeof(TX) == 1 ? 16 * q + 8 * half : 32 * half + 8 * q; }

// A tile of 32 rows by 16 RT ranks, and a part of the reduction.  The four wavefronts take its steps of 64 elements in turn
// and add up in LDS.  Several steps' loads are issued before the first one's products: a wavefront waits for memory
// once per batch.  Bound by memory: 4096 rows of 11008 columns of bfloat16, 16 ranks, 22 us for 90 MB (4.1 TB/s), collected 24;
// 4096 x 4096 codes 11 us, collected 12.6.  Matrix instructions of 32 rows, no transposition, no row in LDS: a lane's eight elements of a
// row are what an instruction takes from it.
template <typename TX, typename TW, int RT, int SPAN, bool VEC, bool ODD>
__global__ __launch_bounds__(256) void k_adapter_first(FirstArgs a)
{
    constexpr int kBatch = (sizeof(TW) == 2 && !(ODD && RT == 4)) || RT == 1 ? 2 : 1;
    constexpr bool kOddX = ODD && sizeof(TX) < 4, kOddW = ODD && sizeof(TW) < 4;
    typedef typename Vec8<TX>::type XV;
    typedef typename Vec8<TW>::type WV;
    __shared__ float sums[4][kRows][16 * RT];
    __shared__ int list[kRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    const unsigned spans = gridDim.x / a.turns;        // turns outermost: the later ones may have no tile, and the chip's eight dies
    const int64_t row0 = (int64_t)(blockIdx.x % spans) * SPAN;     // take workgroups in turn
    const int turn = blockIdx.x / spans, r0 = blockIdx.y * 16 * RT;
    const int64_t k0 = (int64_t)blockIdx.z * a.chunk, k1 = min(k0 + a.chunk, a.K);
    float *out = a.out + (int64_t)blockIdx.z * a.rows * a.R + row0 * a.R;

    Tiles<kRows, SPAN> of;
    of.load(a.ids, row0, a.rows);
    of.start(row0, a.rows, a.adapters, -1);
    if (turn == 0) {                                   // rows without an adapter
#pragma unroll
        for (int g = 0; g < of.kGroups; ++g)
            if (g == wave && of.id[g] == -1)
                for (int r = r0; r < min(r0 + 16 * RT, a.R); ++r) out[(64 * g + lane) * a.R + r] = 0.0f;
    }
    for (int tile = turn; of.seek(tile); tile += a.turns) {
        const int adapter = of.adapter, size = of.size(tile);
        __syncthreads();                               // the last tile's list and sums are read
        of.rows(tile, list, 4);
        __syncthreads();
        const TX *xr[2];
        const TW *wr[RT];
#pragma unroll
        for (int m = 0; m < 2; ++m) xr[m] = (const TX *)a.x + (row0 + list[min(16 * m + l, size - 1)]) * a.stride;
#pragma unroll
        for (int n = 0; n < RT; ++n) wr[n] = (const TW *)a.w + ((int64_t)adapter * a.R + min(r0 + 16 * n + l, a.R - 1)) * a.K;
        int xs[2], ws[RT];
#pragma unroll
        for (int m = 0; m < 2; ++m) xs[m] = shift_of<TX, ODD>(xr[m]);
#pragma unroll
        for (int n = 0; n < RT; ++n) ws[n] = shift_of<TW, ODD>(wr[n]);
        const float scale = a.scale[adapter];
        v4f acc[2][RT];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < RT; ++n) acc[m][n] = v4f(0);
        // `count` steps of this wavefront's from k on; `whole`: all of them lie inside the part
        auto batch = [&](int64_t k, auto whole, auto count) {
            constexpr int kCount = count;
            XV x[kCount][2][2];
            WV w[kCount][2][RT];
            Loaded<TX, kOddX> xl[kCount][2][2];
            Loaded<TW, kOddW> wl[kCount][2][RT];
#pragma unroll
            for (int b = 0; b < kCount; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int64_t c = k + 256 * b + half_at<TX>(q, half);
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        if constexpr (whole) xl[b][half][m].load(dword_of(xr[m], xs[m]), xs[m], c);
                        else x[b][half][m] = columns8<TX, VEC>(xr[m], c, a.K);
                    }
#pragma unroll
                    for (int n = 0; n < RT; ++n) {
                        if constexpr (whole) wl[b][half][n].load(dword_of(wr[n], ws[n]), ws[n], c);
                        else w[b][half][n] = columns8<TW, VEC>(wr[n], c, a.K);
                    }
                }
            loads_first();
            if constexpr (!whole) {
#pragma unroll
                for (int b = 0; b < kCount; ++b)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int64_t c = k + 256 * b + half_at<TX>(q, half);
#pragma unroll
                        for (int m = 0; m < 2; ++m) x[b][half][m] = only<TX, VEC>(x[b][half][m], c, k1, a.K);
#pragma unroll
                        for (int n = 0; n < RT; ++n) w[b][half][n] = only<TW, VEC>(w[b][half][n], c, k1, a.K);
                    }
            }
#pragma unroll
            for (int b = 0; b < kCount; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const typename Operand<TW>::type xm = operand<TW, TX>(whole ? xl[b][half][m].get(xs[m]) : x[b][half][m]);
#pragma unroll
                        for (int n = 0; n < RT; ++n)
                            acc[m][n] = multiply(xm, whole ? wl[b][half][n].get(ws[n]) : w[b][half][n], acc[m][n]);
                    }
        };
        int64_t k = k0 + 64 * wave;
        // A step that is left over by itself, or in a batch that is not whole.  By itself takes another copy of the products: of codes,
        // whose parts are one batch or one step, that costs more than it saves (2070 rows of 4096 columns 7.7 us, 7.0 without; rows of
        // 9360 columns in 16 bits 12.1, 14.4 without).
        typedef std::integral_constant<int, sizeof(TX) == 1 ? kBatch : 1> Rest;
        if constexpr (VEC) {
            for (; k + 256 * (kBatch - 1) + 64 <= k1; k += 256 * kBatch) batch(k, std::true_type(), std::integral_constant<int, kBatch>());
            if (Rest() < kBatch && k + 64 <= k1) {
                batch(k, std::true_type(), Rest());
                k += 256;
            }
        }
        for (; k < k1; k += 256 * Rest()) batch(k, std::false_type(), Rest());
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int n = 0; n < RT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) sums[wave][16 * m + 4 * q + i][16 * n + l] = acc[m][n][i];
        __syncthreads();
        for (int i = threadIdx.x; i < kRows * 16 * RT; i += 256) {
            const int at = i / (16 * RT), col = i % (16 * RT);
            if (at >= size || r0 + col >= a.R) continue;
            const int row = list[at];
            const float s = (sums[0][at][col] + sums[1][at][col]) + (sums[2][at][col] + sums[3][at][col]);
            out[row * a.R + r0 + col] = s * (a.step ? scale * a.step[row0 + row] : scale);
        }
    }
}

// --------------------------------------------------------------------------
// products of H
// --------------------------------------------------------------------------
// The second and the outer products multiply H, which stays in binary32, with elements of a narrower type.  Sixteen reduction
// elements of 16 rows by 128 columns: a lane holds eight neighbouring columns of each of its four elements, so a matrix
// instruction j of eight takes everyone's column j, neither operand needs a transposition, and loads and stores are vectors.
//   bfloat16 and codes: h is the sum of three bfloat16 (its leading, middle and last eight bits, cut off: exact), so three
//     instructions of sixteen elements give the products of binary32 in 48 cycles a column; infinite elements come out as NaN
//   others: four binary32 instructions of four elements, 128 cycles
template <typename T> constexpr bool in_thirds = std::is_same<T, bf16>::value || std::is_same<T, int8_t>::value;
// Which of the sixteen elements a lane of quarter q holds as its i-th.
template <typename T> __device__ inline int element_of(int q, int i) { return in_thirds<T> ? 4 * q + i : 4 * i + q; }

typedef short v4s __attribute__((ext_vector_type(4)));
struct Thirds { uint32_t w[3][2]; };   // two elements to a word

__device__ inline uint32_t upper_halves(uint32_t second, uint32_t first) { return __builtin_amdgcn_perm(second, first, 0x07060302u); }
__device__ inline uint32_t lower_halves(uint32_t second, uint32_t first) { return __builtin_amdgcn_perm(second, first, 0x05040100u); }
// The part of h that its first eight bits leave.
__device__ inline float rest(float h)
{
    const float top = __uint_as_float(__float_as_uint(h) & 0xffff0000u);
    return top == h ? 0.0f : h - top;
}
__device__ inline Thirds thirds(const float (&h)[4])
{
    Thirds t;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = h[i];
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        t.w[p][0] = upper_halves(__float_as_uint(v[1]), __float_as_uint(v[0]));
        t.w[p][1] = upper_halves(__float_as_uint(v[3]), __float_as_uint(v[2]));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = rest(v[i]);
    }
    return t;
}
__device__ inline v4s words(uint32_t a, uint32_t b)
{
    union { uint32_t w[2]; v4s v; } u = {{a, b}};
    return u.v;
}
// Eight bfloat16 as four words.
__device__ inline void as_words(v8bf v, uint32_t (&w)[4]) { __builtin_memcpy(w, &v, 16); }
__device__ inline void as_words(v2u v, uint32_t (&w)[4])
{
    const v8f f = widen(v);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = upper_halves(__float_as_uint(f[2 * j + 1]), __float_as_uint(f[2 * j]));
}

// H of a lane's row and elements, and the columns of x, as the instructions take them.
template <typename T, bool THIRDS = in_thirds<T>> struct H16 {
    Thirds t;
    __device__ H16(const float (&h)[4]) : t(thirds(h)) {}
};
template <typename T> struct H16<T, false> {
    float v[4];
    __device__ H16(const float (&h)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = h[i];
    }
};
template <typename T, bool THIRDS = in_thirds<T>> struct Columns {
    uint32_t w[4][4];
    __device__ Columns(const typename Vec8<T>::type (&x)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) as_words(x[i], w[i]);
    }
};
template <typename T> struct Columns<T, false> {
    typename Vec8<T>::type v[4];
    __device__ Columns(const typename Vec8<T>::type (&x)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = x[i];
    }
};
// y[j] += sum over the sixteen elements of h times column j0 + j.
template <typename T, int N> __device__ inline void product16(const H16<T, true> &h, const Columns<T, true> &x, int j0, v4f (&y)[N])
{
#pragma unroll
    for (int p = 2; p >= 0; --p)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int d = (j0 + j) / 2;
            const v4s c = j & 1 ? words(upper_halves(x.w[1][d], x.w[0][d]), upper_halves(x.w[3][d], x.w[2][d]))
                                : words(lower_halves(x.w[1][d], x.w[0][d]), lower_halves(x.w[3][d], x.w[2][d]));
            y[j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(words(h.t.w[p][0], h.t.w[p][1]), c, y[j], 0, 0, 0);
        }
}
template <typename T, int N> __device__ inline void product16(const H16<T, false> &h, const Columns<T, false> &x, int j0, v4f (&y)[N])
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(h.v[i], widen(x.v[i][j0 + j]), y[j], 0, 0, 0);
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
    bool has_base;                     // else base is memory that can be read as a row of C elements, its stride 0
    int R, splits, adapters, out_type;
    int turns, walks;                  // workgroups that share a span's tiles, and the columns of a tile
};

// A wavefront does 16 rows by 128 columns.  The ranks come sixteen at a time, their products added to the row's sum where the
// row has the adapter.  A workgroup walks along its rows, H in LDS; the next tile's base and W are on their way while one is
// computed and stored.  Rows and adapters are buffers of their own length: ranks beyond R read as 0, rows beyond the last are not
// written, and an address is one register of a lane's.  Bound by memory: 4096 x 4096, 16 ranks, binary32 base and bfloat16 out 22 us for
// 101 MB (4.6 TB/s); 2048 x 4096, 64 ranks, base and out in binary32 23 us for 67 MB, and each tile's 512 KB of W from L2 (21
// without the products).
constexpr int kSecondRows = 16;
__host__ __device__ inline int second_pitch(int R) { return (R + 15) / 16 * 16 + 1; }

// Eight columns at once or one by one, from a byte offset on.
template <typename T, bool VEC> __device__ inline typename Vec8<T>::type buffer_columns(__amdgpu_buffer_rsrc_t b, int offset)
{
    if constexpr (VEC) return buffer_load8<T>(b, offset);
    else {
        union { typename Vec8<T>::type v; T e[8]; } u;
#pragma unroll
        for (int i = 0; i < 8; ++i) u.e[i] = buffer_load1<T>(b, offset + i * (int)sizeof(T));
        return u.v;
    }
}
// Of eight columns those from the first `skip` on, and at most `columns`; of a row that is not `there` none.
template <typename T, bool VEC>
__device__ inline void store_tile(__amdgpu_buffer_rsrc_t b, int offset, int skip, int columns, bool there, v8f v)
{
    if (VEC && skip == 0 && there) buffer_store8<T>(b, offset, __builtin_convertvector(v, typename Vec8<T>::type));
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i >= skip && i < columns && there) buffer_store1<T>(b, offset + i * (int)sizeof(T), (T)v[i]);
    }
}

// H of a tile into LDS, its parts added up in order: four elements of a thread and four parts under way.  Sixteen ranks of a row are
// neighbours, then the rows, then the next sixteen ranks.  `row_of` gives the tile's rows, some row beyond the last `n`.
template <class RowOf> __device__ inline void load_h(const SecondArgs &a, float *hs, int n, bool keep, RowOf row_of)
{
    const int pitch = second_pitch(a.R);
    for (int i = threadIdx.x; i - (int)threadIdx.x < kSecondRows * (pitch - 1); i += 4 * blockDim.x) {
        int row[4], r[4];
        int64_t at[4];
        float sum[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = i + j * blockDim.x;
            row[j] = (e >> 4) % kSecondRows;
            r[j] = e / (16 * kSecondRows) * 16 + (e & 15);
            at[j] = row_of(row[j]) * a.R + min(r[j], a.R - 1);
            sum[j] = 0.0f;
        }
        for (int p = 0; p < a.splits; p += 4) {
            float v[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[k][j] = a.h[min(p + k, a.splits - 1) * a.rows * a.R + at[j]];
            loads_first();
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] += p + k < a.splits ? v[k][j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (r[j] >= pitch - 1) continue;
            if (r[j] < a.R && keep && a.h_out && row[j] < n) a.h_out[at[j]] = sum[j];
            hs[row[j] * pitch + r[j]] = r[j] < a.R ? sum[j] : 0.0f;
        }
    }
}

template <typename TW, typename TB, bool VEC> __global__ __launch_bounds__(256, 2) void k_adapter_second(SecondArgs a)
{
    typedef typename Vec8<TW>::type WV;
    typedef typename Vec8<TB>::type BV;
    extern __shared__ float hs[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x / 64, l = lane & 15, q = lane >> 4;
    const int64_t row0 = (int64_t)(blockIdx.x / a.walks) * kSecondRows;
    const int walk = blockIdx.x % a.walks, pitch = second_pitch(a.R), C = (int)a.C;
    const int tiles = (C + 127) / 128, stride = a.walks * waves;
    int tile = walk * waves + wave;                    // of 128 columns

    const uint32_t rows = (uint32_t)min((int64_t)kSecondRows, a.rows - row0);
    const int base_pitch = (int)a.base_stride * (int)sizeof(TB), out_size = a.out_type == PWLQ_F32 ? 4 : (int)sizeof(TW);
    const int out_pitch = (int)a.out_stride * out_size;
    const __amdgpu_buffer_rsrc_t base_rows = row_buffer((const TB *)a.base + row0 * a.base_stride, (rows - 1) * base_pitch + C * sizeof(TB));
    const __amdgpu_buffer_rsrc_t out_rows =
        row_buffer((char *)a.out + row0 * a.out_stride * out_size, (rows - 1) * out_pitch + C * out_size);

    // a lane's first column in a tile; the last vector of a row that is no whole number of them starts further left
    auto column = [&](int tile) { return VEC ? (int)start_of(128 * tile + 8 * l, C) : 128 * tile + 8 * l; };
    // what a tile needs from memory: base, and the first adapter's first ranks
    BV base[4];
    WV w[4];
    auto load_base = [&](int tile) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            base[i] = buffer_columns<TB, VEC>(base_rows, (4 * q + i) * base_pitch + column(tile) * (int)sizeof(TB));
    };
    auto load_ranks = [&](int adapter, int r0, int tile) {
        const __amdgpu_buffer_rsrc_t b = row_buffer((const TW *)a.w + (int64_t)adapter * a.R * C, (uint32_t)a.R * C * sizeof(TW));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = buffer_columns<TW, VEC>(b, (int)((uint32_t)((r0 + element_of<TW>(q, i)) * (uint32_t)C + column(tile)) * (uint32_t)sizeof(TW)));
    };
    const int id = Adapters::load(a.ids, row0, a.rows);
    float factor[4];                                   // without factors any number that can be read
    const float *from = a.base_step ? a.base_step : a.h;
#pragma unroll
    for (int i = 0; i < 4; ++i) factor[i] = from[a.base_step ? clamp_row(row0 + 4 * q + i, a.rows) : 0];
    load_base(tile);
    loads_first();
    const Adapters all(id, row0, a.rows, a.adapters, kSecondRows);
    Adapters of = all;
    int adapter = 0;
    uint64_t mine = 0;
    of.next(adapter, mine);
    const int first_adapter = adapter;
    load_ranks(adapter, 0, tile);

    load_h(a, hs, rows, walk == 0, [&](int row) { return clamp_row(row0 + row, a.rows); });
    __syncthreads();
    for (; tile < tiles; tile += stride) {
        v8f acc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = a.has_base ? widen(base[i]) * (a.base_step ? factor[i] : 1.0f) : v8f(0);
        const int after = tile + stride < tiles ? tile + stride : tile;
        load_base(after);
        of = all;
        bool more = of.next(adapter, mine);
        int r0 = 0;
        while (more) {
            WV now[4];
            float h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                now[i] = w[i];
                h[i] = hs[l * pitch + r0 + element_of<TW>(q, i)];
            }
            const uint64_t own_rows = mine;
            r0 += 16;
            if (r0 >= a.R) {
                r0 = 0;
                more = of.next(adapter, mine);
            }
            load_ranks(more ? adapter : first_adapter, r0, more ? tile : after);
            loads_first();
            const H16<TW> h16(h);
            const Columns<TW> columns(now);
#pragma unroll
            for (int j0 = 0; j0 < 8; j0 += 4) {        // four columns' sums at a time
                v4f y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = v4f(0);
                product16(h16, columns, j0, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool own = (own_rows >> (4 * q + i)) & 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j0 + j] += own ? y[j][i] : 0.0f;
                }
                loads_first();
            }
        }
        const int offset = 4 * q * out_pitch + column(tile) * out_size, left = C - column(tile);
        const int skip = VEC ? beyond(128 * tile + 8 * l, C) : 0;
        if (a.out_type == PWLQ_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) store_tile<float, VEC>(out_rows, offset + i * out_pitch, skip, left, true, acc[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) store_tile<TW, VEC>(out_rows, offset + i * out_pitch, skip, left, true, acc[i]);
        }
    }
}

// The same for tiles that are collected, a tile's rows of one adapter: what the ranks give is added to the base by the products.
// 4096 x 4096, 16 ranks, 8 adapters, binary32 base and bfloat16 out 26.5 us; rows, ids and their list come one after the other at
// a tile's start, and the tiles that further adapters begin leave some workgroups with two.
template <typename TW, typename TB, bool VEC> __global__ __launch_bounds__(256, 2) void k_adapter_second_collected(SecondArgs a)
{
    typedef typename Vec8<TW>::type WV;
    typedef typename Vec8<TB>::type BV;
    extern __shared__ float hs[];
    __shared__ int list[kSecondRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x / 64, l = lane & 15, q = lane >> 4;
    const unsigned spans = gridDim.x / (a.turns * a.walks);
    const unsigned span = blockIdx.x % spans;          // turns outermost: the later ones may have no tile
    const int walk = blockIdx.x / spans % a.walks, turn = blockIdx.x / (spans * a.walks), pitch = second_pitch(a.R), C = (int)a.C;
    const int64_t row0 = (int64_t)span * kCollected;
    const int tiles = (C + 127) / 128, stride = a.walks * waves;      // tiles of 128 columns

    const int rows = (int)min((int64_t)kCollected, a.rows - row0);
    const int base_pitch = (int)a.base_stride * (int)sizeof(TB), out_size = a.out_type == PWLQ_F32 ? 4 : (int)sizeof(TW);
    const int out_pitch = (int)a.out_stride * out_size;
    const __amdgpu_buffer_rsrc_t base_rows = row_buffer((const TB *)a.base + row0 * a.base_stride, (uint32_t)(rows - 1) * base_pitch + C * sizeof(TB));
    const __amdgpu_buffer_rsrc_t out_rows =
        row_buffer((char *)a.out + row0 * a.out_stride * out_size, (uint32_t)(rows - 1) * out_pitch + C * out_size);
    // a lane's first column in a tile; the last vector of a row that is no whole number of them starts further left
    auto column = [&](int tile) { return VEC ? (int)start_of(128 * tile + 8 * l, C) : 128 * tile + 8 * l; };

    int row[4];                                        // the lane's rows of the tile
    float factor[4];                                   // without factors any number that can be read
    BV base[4];
    WV w[4];
    auto load_base = [&](int tile) {
#pragma unroll
        for (int i = 0; i < 4; ++i) base[i] = buffer_columns<TB, VEC>(base_rows, row[i] * base_pitch + column(tile) * (int)sizeof(TB));
    };
    const float *factors = a.base_step ? a.base_step + row0 : a.h;
    Tiles<kSecondRows, kCollected> of;
    of.load(a.ids, row0, a.rows);
    of.start(row0, a.rows, a.adapters, -2);
    for (int at = turn; of.seek(at); at += a.turns) {
        const int adapter = of.adapter, n = of.size(at);
        int tile = walk * waves + wave;
        __syncthreads();                               // the last tile's list and H are read
        of.rows(at, list, waves);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            row[i] = list[min(4 * q + i, n - 1)];
            factor[i] = factors[a.base_step ? row[i] : 0];
        }
        load_base(tile);
        const __amdgpu_buffer_rsrc_t ranks = row_buffer((const TW *)a.w + (int64_t)max(adapter, 0) * a.R * C, (uint32_t)a.R * C * sizeof(TW));
        auto load_ranks = [&](int r0, int tile) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = buffer_columns<TW, VEC>(ranks, (int)((uint32_t)((r0 + element_of<TW>(q, i)) * (uint32_t)C + column(tile)) * (uint32_t)sizeof(TW)));
        };
        load_ranks(0, tile);

        load_h(a, hs, n, walk == 0, [&](int i) { return row0 + list[min(i, n - 1)]; });
        __syncthreads();
        for (; tile < tiles; tile += stride) {
            v4f acc[2][4];                             // of a column: the lane's four rows; four columns at a time
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v8f b = a.has_base ? widen(base[i]) * (a.base_step ? factor[i] : 1.0f) : v8f(0);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j / 4][j % 4][i] = b[j];
            }
            const int after = tile + stride < tiles ? tile + stride : tile;
            load_base(after);                          // the next columns'
            for (int r0 = 0; r0 < a.R && adapter >= 0; r0 += 16) {
                WV now[4];
                float h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    now[i] = w[i];
                    h[i] = hs[l * pitch + r0 + element_of<TW>(q, i)];
                }
                const bool last = r0 + 16 >= a.R;
                load_ranks(last ? 0 : r0 + 16, last ? after : tile);
                loads_first();
                const H16<TW> h16(h);
                const Columns<TW> columns(now);
                product16(h16, columns, 0, acc[0]);
                loads_first();
                product16(h16, columns, 4, acc[1]);
                loads_first();
            }
            const int left = C - column(tile), skip = VEC ? beyond(128 * tile + 8 * l, C) : 0;
            const int offset = column(tile) * out_size;
            v8f v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = acc[j / 4][j % 4][i];
            if (a.out_type == PWLQ_F32) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    store_tile<float, VEC>(out_rows, row[i] * out_pitch + offset, skip, left, 4 * q + i < n, v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    store_tile<TW, VEC>(out_rows, row[i] * out_pitch + offset, skip, left, 4 * q + i < n, v[i]);
            }
        }
    }
}

// --------------------------------------------------------------------------
// both products for few rows
// --------------------------------------------------------------------------
// Eight columns in their places: those of a shifted vector that belong to the lane before are left out.
template <bool VEC> __device__ inline void put_columns(v8f &place, v8f y, int64_t col, int64_t cols)
{
    const int skip = VEC ? beyond(col, cols) : 0;
    if (skip == 0) place = y;
    else {
#pragma unroll
        for (int j = 1; j < 8; ++j)
            if (j >= skip) ((float *)&place)[j - skip] = y[j];
    }
}

// Both products of one row in one launch, for 512 columns: the row's H is computed by each of its workgroups anew, which costs
// reading down again from L2 but no second launch and no wait for it.  The sixteen wavefronts share the ranks of both products.
// Bound by latency: a wavefront's eight loads of x and down, the sum, up, the sum of the wavefronts, 6.0 us for one row of 4096 x 4096
// with 16 ranks and 6.5 for eight of 4096 x 11008.
struct TokenArgs {
    const void *x, *down, *up, *base;
    void *out;
    int64_t x_stride, base_stride, out_stride, K, C;
    const float *x_step, *base_step, *scale;
    const int32_t *ids;
    float *h;
    int R, adapters, base_type, out_type;
};
constexpr int kTokenThreads = 1024, kTokenColumns = 512, kTokenWaves = kTokenThreads / 64, kTokenRanks = 48;

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
        const WV ahead = columns8<TW, VEC>(up + (int64_t)min(wave, a.R - 1) * a.C, col, a.C);
        const TX *x = (const TX *)a.x + row * a.x_stride;
        const float scale = a.x_step ? a.scale[id] * a.x_step[row] : a.scale[id];
        for (int r = wave; r < a.R; r += kTokenWaves) {
            const TW *w = (const TW *)a.down + ((int64_t)id * a.R + r) * a.K;
            v8f t = v8f(0);
            if constexpr (VEC) {
                const int64_t whole = a.K / 8;         // vectors; those beyond are read from the last one and count nothing
                for (int64_t k = 0; k < whole; k += 64 * kAhead) {
                    XV xv[kAhead];
                    WV wv[kAhead];
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const int64_t c = 8 * min(k + 64 * i + lane, whole - 1);
                        xv[i] = load8(x + c);
                        wv[i] = load8(w + c);
                    }
                    loads_first();
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        const v8f p = widen(xv[i]) * widen(wv[i]);
                        t += k + 64 * i + lane < whole ? p : v8f(0);
                    }
                }
                if (8 * whole + lane < a.K) t[0] += widen(x[8 * whole + lane]) * widen(w[8 * whole + lane]);
            } else {
                for (int64_t k = lane; k < a.K; k += 64) t[0] += widen(x[k]) * widen(w[k]);
            }
            const float s = wave_sum(((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7])));
            if (lane == 0) hs[r] = s * scale;
        }
        __syncthreads();
        if (blockIdx.x == 0 && threadIdx.x < a.R) a.h[row * a.R + threadIdx.x] = hs[threadIdx.x];
        if (wave < a.R) y = hs[wave] * widen(ahead);
        for (int r = wave + kTokenWaves; r < a.R; r += kTokenWaves) y += hs[r] * widen(columns8<TW, VEC>(up + (int64_t)r * a.C, col, a.C));
    } else if (blockIdx.x == 0 && threadIdx.x < a.R) {
        a.h[row * a.R + threadIdx.x] = 0.0f;
    }
    put_columns<VEC>(sums[wave][lane], y, col, a.C);
    __syncthreads();
    if (threadIdx.x >= kTokenColumns || col0 + threadIdx.x >= a.C) return;
    float s = 0.0f;
#pragma unroll
    for (int g = 0; g < kTokenWaves; ++g) s += ((const float *)sums[g])[threadIdx.x];
    const int64_t at = row * a.out_stride + col0 + threadIdx.x;
    if (a.out_type == PWLQ_F32) ((float *)a.out)[at] = base + s;
    else ((TW *)a.out)[at] = (TW)(base + s);
}

// The second product of a few rows, each by itself: 512 columns of a row, the four wavefronts share the ranks.  Tiles of sixteen
// rows would do their adapters one after the other.  250 x 1000, 5 ranks, 3 adapters 4.3 us, by tiles 6.1.
template <typename TW, bool VEC>
__global__ __launch_bounds__(256) void k_adapter_second_row(SecondArgs a, int base_type)
{
    __shared__ float hs[256];
    __shared__ v8f sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = blockIdx.y, col0 = (int64_t)blockIdx.x * 512, col = col0 + 8 * lane;
    const int id = a.ids[row];
    const bool any = id >= 0 && id < a.adapters;
    float base[2];
    if (a.has_base) {
        const float factor = a.base_step ? a.base_step[row] : 1.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t at = row * a.base_stride + min(col0 + threadIdx.x + 256 * i, a.C - 1);
            base[i] = (base_type == PWLQ_F32 ? ((const float *)a.base)[at] : widen(((const TW *)a.base)[at])) * factor;
        }
    } else {
        base[0] = base[1] = 0.0f;
    }
    if ((int)threadIdx.x < a.R) {
        float s = 0.0f;
        for (int p = 0; p < a.splits; ++p) s += a.h[(p * a.rows + row) * a.R + threadIdx.x];
        hs[threadIdx.x] = s;
        if (blockIdx.x == 0 && a.h_out) a.h_out[row * a.R + threadIdx.x] = s;
    }
    __syncthreads();
    v8f y = v8f(0);
    if (any) {
        const TW *w = (const TW *)a.w + (int64_t)id * a.R * a.C;
        for (int r = wave; r < a.R; r += 16) {             // four ranks under way
            typename Vec8<TW>::type v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = columns8<TW, VEC>(w + (int64_t)min(r + 4 * j, a.R - 1) * a.C, col, a.C);
            loads_first();
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (r + 4 * j < a.R) y += hs[r + 4 * j] * widen(v[j]);
        }
    }
    put_columns<VEC>(sums[wave][lane], y, col, a.C);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = threadIdx.x + 256 * i;
        if (col0 + c >= a.C) return;
        const float s = (((const float *)sums[0])[c] + ((const float *)sums[1])[c]) + (((const float *)sums[2])[c] + ((const float *)sums[3])[c]);
        const int64_t at = row * a.out_stride + col0 + c;
        if (a.out_type == PWLQ_F32) ((float *)a.out)[at] = base[i] + s;
        else ((TW *)a.out)[at] = (TW)(base[i] + s);
    }
}

// --------------------------------------------------------------------------
// outer products
// --------------------------------------------------------------------------
struct OuterArgs {
    const float *h;                    // [rows, R]
    const void *x;
    int64_t stride, rows, C, span;     // span: rows of a workgroup
    const float *step;
    const int32_t *ids;
    int R, adapters, column_tiles, rank_blocks, slots;
    float *out;                        // [splits, adapters, R, C]
    int32_t *present;                  // [splits, adapters]: whether the part has rows of the adapter; NULL where there is one part
    bool flags;                        // whether this product writes them: both have the same rows
};

// 16 RT ranks by 128 columns of the adapters' gradients, over a part of the rows: for each adapter that has some of them, one
// after the other.  Its rows are listed in LDS first, 512 at a time, so that no other row is read; the four wavefronts take
// sixteen of them each in turn, the next ones' loads under way, and add up in LDS.  Bound by memory and, at 64 ranks, by the matrix
// instructions' thirds: 4096 rows, 4096 codes and 11008 columns of bfloat16, 16 ranks 26 us for 107 MB (4.1 TB/s); 2048 rows, 4096 codes
// and 4096 columns of bfloat16, 64 ranks 21.3 us, each of its two passes over 32 ranks reading the rows again.  With binary32 weights and
// more than 16 ranks 12 to 36 registers spill.
constexpr int kListed = 512;

template <int RT> struct OuterLds {
    v4f sums[2][RT * 8][64];
    int list[kListed];
};

// `slot`: of a.slots (a power of two) workgroups that share the adapters of these rows, by their lowest bits.
template <typename TX, int RT, bool VEC> __device__ inline void outer_tile(const OuterArgs &a, int tile, int split, int slot, OuterLds<RT> &lds)
{
    typedef typename Vec8<TX>::type XV;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & 15, q = lane >> 4;
    const int64_t col = (int64_t)(tile % a.column_tiles) * 128 + 8 * l;
    const int r0 = tile / a.column_tiles * 16 * RT;
    const int64_t t0 = split * a.span, t1 = min(t0 + a.span, a.rows);
    struct Rows {
        XV x[4];
        float h[4][RT], step[4];
    };
    float *const part = a.out + (int64_t)split * a.adapters * a.R * a.C;
    int32_t *const present = a.present && a.flags && tile == 0 ? a.present + (int64_t)split * a.adapters : nullptr;
    if (present)
        for (int i = slot + threadIdx.x * a.slots; i < a.adapters; i += 256 * a.slots) present[i] = 0;
    v4f acc[RT][8];
    for (int adapter = slot - a.slots, next;; adapter = next) {
        next = a.adapters;
        bool alone = true;                             // the first wavefront has all rows
#pragma unroll
        for (int n = 0; n < RT; ++n)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[n][j] = v4f(0);
        for (int64_t t = t0; t < t1; t += kListed) {
            int id[kListed / 64];
#pragma unroll
            for (int g = 0; g < kListed / 64; ++g) id[g] = a.ids[clamp_row(t + 64 * g + lane, t1)];
            loads_first();
#pragma unroll
            for (int g = 0; g < kListed / 64; ++g)
                if (id[g] > adapter && (id[g] & (a.slots - 1)) == slot) next = min(next, id[g]);
            if (adapter < 0) continue;
            int count = 0;
            __syncthreads();
#pragma unroll
            for (int g = 0; g < kListed / 64; ++g) {
                const uint64_t mine = __ballot(id[g] == adapter && t + 64 * g + lane < t1);
                if (g % 4 == wave && ((mine >> lane) & 1)) lds.list[count + __builtin_popcountll(mine & ((1ull << lane) - 1))] = 64 * g + lane;
                count += __builtin_popcountll(mine);
            }
            __syncthreads();
            alone &= count <= 16;
            auto load = [&](int first, Rows &v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t row = t + lds.list[min(first + element_of<TX>(q, i), count - 1)];
                    v.x[i] = columns8<TX, VEC>((const TX *)a.x + row * a.stride, col, a.C);
#pragma unroll
                    for (int n = 0; n < RT; ++n) v.h[i][n] = a.h[row * a.R + min(r0 + 16 * n + l, a.R - 1)];
                    if constexpr (sizeof(TX) == 1) v.step[i] = a.step[row];
                }
            };
            int first = 16 * wave;
            if (first >= count) continue;
            // one step ahead with sixteen ranks, whose workgroups are four to a CU, two steps ahead with 32 (two to a CU);
            // beyond the list its last row is read and not used
            Rows now, after, later;
            load(first, now);
            if (RT > 1) load(first + 64, after);
            for (; first < count; first += 64) {
                load(first + 64 * RT, RT > 1 ? later : after);
                loads_first();
                bool own[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    own[i] = first + element_of<TX>(q, i) < count;
                    now.x[i] = own[i] ? now.x[i] : XV(0);
                }
                const Columns<TX> columns(now.x);
#pragma unroll
                for (int n = 0; n < RT; ++n) {
                    float h[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        h[i] = now.h[i][n];
                        if constexpr (sizeof(TX) == 1) h[i] *= now.step[i];
                        h[i] = own[i] ? h[i] : 0.0f;
                    }
                    product16(H16<TX>(h), columns, 0, acc[n]);
                }
                now = after;
                if (RT > 1) after = later;
            }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) next = min(next, __shfl_xor(next, d));
        next = __builtin_amdgcn_readfirstlane(next);
        // adapters without rows here: nothing in a part, zeros where there are no parts
        if (!a.present)
            for (int none = adapter + a.slots; none < next; none += a.slots)
                for (int i = threadIdx.x; i < 16 * RT * 128; i += 256) {
                    const int r = r0 + i / 128;
                    const int64_t c = (int64_t)(tile % a.column_tiles) * 128 + i % 128;
                    if (r < a.R && c < a.C) part[((int64_t)none * a.R + r) * a.C + c] = 0.0f;
                }
        if (adapter >= 0) {
            if (present && (int)threadIdx.x == adapter / a.slots % 256) present[adapter] = 1;
            if (!alone) {
                if (wave >= 2) {
#pragma unroll
                    for (int n = 0; n < RT; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j) lds.sums[wave - 2][8 * n + j][lane] = acc[n][j];
                }
                __syncthreads();
                if (wave < 2) {
#pragma unroll
                    for (int n = 0; n < RT; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j) acc[n][j] += lds.sums[wave][8 * n + j][lane];
                }
                __syncthreads();
                if (wave == 1) {
#pragma unroll
                    for (int n = 0; n < RT; ++n)
#pragma unroll
                        for (int j = 0; j < 8; ++j) lds.sums[0][8 * n + j][lane] = acc[n][j];
                }
                __syncthreads();
            }
            if (wave == 0) {
                float *out = part + (int64_t)adapter * a.R * a.C;
#pragma unroll
                for (int n = 0; n < RT; ++n) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (!alone) acc[n][j] += lds.sums[0][8 * n + j][lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = r0 + 16 * n + 4 * q + i;
                        v8f v;
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = acc[n][j][i];
                        if (r >= a.R) continue;
                        if constexpr (VEC) {
                            if (col < a.C) store8(out + (int64_t)r * a.C + start_of(col, a.C), v);     // columns of two vectors: the same sums twice
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (col + j < a.C) out[(int64_t)r * a.C + col + j] = v[j];
                        }
                    }
                }
            }
        }
        if (next >= a.adapters) return;
    }
}

// Both gradients in one launch: the second fills the chip while the first one's last workgroups end.
template <typename TX, typename TY, int RT, bool VEC>
__global__ __launch_bounds__(256, RT == 1 && VEC && sizeof(TY) == 2 ? 4 : 2) void k_adapter_outer(OuterArgs up, OuterArgs down)
{
    __shared__ OuterLds<RT> lds;
    const int ups = up.column_tiles * up.rank_blocks;
    if ((int)blockIdx.x < ups) outer_tile<TY, RT, VEC>(up, blockIdx.x, blockIdx.y, blockIdx.z, lds);
    else outer_tile<TX, RT, VEC>(down, blockIdx.x - ups, blockIdx.y, blockIdx.z, lds);
}

// Parts of both gradients added up in order: 5.2 us for 8 parts of 15104 columns by 16 ranks of four adapters, of which only those that
// have rows in a part are read.
struct JoinArgs {
    const float *part[2];
    const int32_t *present;
    float *out[2];
    int64_t each[2];                   // R C
    int splits, adapters;
};
__global__ __launch_bounds__(256) void k_adapter_join(JoinArgs a)
{
    const int which = blockIdx.z, adapter = blockIdx.y, lane = threadIdx.x & 63;
    const int64_t each = a.each[which], n = each * a.adapters;
    const float *part = a.part[which] + adapter * each;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i - lane < each; i += (int64_t)gridDim.x * 256) {
        const int64_t at = min(i, each - 1);
        float s = 0.0f;
        for (int p0 = 0; p0 < a.splits; p0 += 64) {
            uint64_t parts = __ballot(p0 + lane < a.splits && a.present[(p0 + lane) * a.adapters + adapter]);
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

int rank_tiles(int R) { return R <= 16 ? 1 : R <= 32 ? 2 : 4; }
int rank_blocks(int R) { return (R + 16 * rank_tiles(R) - 1) / (16 * rank_tiles(R)); }

// Parts of the first product's reduction: workgroups for the whole chip, each with a batch of steps for its wavefronts at least.
// Four to a CU: 4096 rows of 11008 columns 22 us, two to a CU 33, eight 30.
int first_splits(int64_t T, int64_t K, int R)
{
    if (!T) return 1;
    const int64_t wgs = (T + kRows - 1) / kRows * rank_blocks(R);
    return (int)std::max<int64_t>(1, std::min<int64_t>(1024 / wgs, (K + 511) / 512));
}
int64_t first_chunk(int64_t K, int splits) { return ((K + splits - 1) / splits + 255) / 256 * 256; }

// Parts of the rows for the outer products: as many workgroups as are resident, four to a CU up to 16 ranks (25.0 us where two
// take 28.6), two beyond; in blocks of 32 ranks (20.7 us for 64 ranks; of 64 at once 23.3).
int outer_blocks(int R) { return R <= 16 ? 1 : (R + 31) / 32; }
// A part leaves a sum for each adapter that has rows in it, to be written and read again, so a part has 64 rows for each adapter on
// average.  The whole backward pass of 4096 x 4096 of bfloat16, 16 ranks, parts for the whole chip -> these, in us: 534 rows of 32 adapters
// in runs 67 -> 41, alternating 130 -> 50; 4096 rows of 8 adapters 57 -> 56 and 91 -> 73, of 32 85 -> 88 and 254 -> 129, and where
// all the rows have one of the 32 55 -> 71.
// But a part has fewer than 8192 rows, as far as the sums of parts of 4096 fit 4 GiB: each of its workgroups walks all of it for the adapters of
// its slot, and a large bank may have few in use.  One part -> these, of 512 adapters: 32768 rows of one 703 -> 383, in runs of all
// 3119 -> 868, alternating among 8 407 -> 471 and among all 6166 -> 6744; 8192 rows of one 226 -> 208, alternating among 8 144 -> 190.
int64_t outer_span(int64_t T, int64_t K, int64_t N, int R, int adapters)
{
    const int64_t wgs = ((K + 127) / 128 + (N + 127) / 128) * outer_blocks(R);
    const int64_t least = std::min<int64_t>(T / 4096, (4LL << 30) / ((int64_t)sizeof(float) * adapters * R * (K + N)));
    const int64_t most = adapters > 1 ? std::max<int64_t>(T / (64 * adapters), least) : (T + 63) / 64;
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>((R <= 16 ? 1024 : 512) / wgs, most));
    return ((T + splits - 1) / splits + 63) / 64 * 64;
}
int outer_splits(int64_t T, int64_t K, int64_t N, int R, int adapters)
{
    const int64_t span = outer_span(T, K, N, R, adapters);
    return (int)((T + span - 1) / span);
}

// Where that leaves CUs idle the adapters are done beside each other.
int outer_slots(int64_t T, int64_t K, int64_t N, int R, int adapters)
{
    const int64_t wgs = ((K + 127) / 128 + (N + 127) / 128) * outer_blocks(R) * outer_splits(T, K, N, R, adapters);
    int slots = 1;
    while (2 * slots <= adapters && 2 * slots * wgs <= 1024) slots *= 2;
    return slots;
}

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
    float *dh, *parts, *down, *up;     // down, up: parts of the gradients; NULL where there is one part
    int32_t *present;
    int splits;
    size_t bytes;
    BackwardSpace(void *workspace, int64_t T, int64_t K, int64_t N, int R, int adapters)
    {
        Carver c = {(char *)workspace};
        const int first = first_splits(T, N, R);
        splits = outer_splits(T, K, N, R, adapters);
        dh = c.take<float>(T * R);
        parts = first > 1 ? c.take<float>(first * T * R) : dh;
        const int64_t all = splits > 1 ? (int64_t)splits * adapters : 0;
        down = c.take<float>(all * R * K);
        up = c.take<float>(all * R * N);
        present = c.take<int32_t>(all);
        bytes = c.at;
    }
};

// Whether rows are collected by adapter from spans of 256: see Tiles.  Collecting takes a longer start (ids, a list, the rows'
// addresses from it) and pays where a tile of neighbouring rows would be done for many adapters, each with many ranks.  Both products
// of 4096 x 4096, 16 ranks, in us, not collected -> collected, rows in runs and rows whose adapters alternate: 256 rows of 2 adapters
// 10.0 -> 11.5 and 10.2 -> 11.5; of 8 adapters 11.4 -> 13.0 and 15.6 -> 13.7; 2048 rows of 8 adapters 21.7 -> 23.4 and 44.9 -> 25.4;
// 4096 rows of 16 adapters 32.2 -> 31.6 and 106 -> 43 (inputs in the caches; with inputs from memory 4096 rows of 8 adapters in runs
// 32 -> 38).  93 rows of 8 adapters and 43 ranks, alternating: 29 -> 21.
bool collected(int64_t rows, int R, int adapters) { return adapters > 1 && rows * adapters * ((R + 15) / 16) >= 2048; }

// Workgroups that share the tiles of a span of `in_span` rows: one for each tile that it has if its rows have one adapter, in a collected
// span some for the tiles that further adapters begin, and more where `fill` of them are wanted, up to the tiles there can be.
int turns(int64_t in_span, int tile, int adapters, bool collect, int64_t fill)
{
    const int64_t whole = (in_span + tile - 1) / tile, most = whole + std::min<int64_t>(adapters, in_span - 1);
    return (int)std::min(most, std::max(whole + (collect ? std::min<int64_t>(adapters, whole / 2) : 0), fill));
}

template <typename TX, typename TW> void first_as(FirstArgs a, bool vec, hipStream_t stream)
{
    const bool collect = collected(a.rows, a.R, a.adapters);
    const int64_t rows = collect ? kCollected : kRows, spans = (a.rows + rows - 1) / rows, splits = (a.K + a.chunk - 1) / a.chunk;
    a.turns = turns(std::min(a.rows, rows), kRows, a.adapters, collect, 2048 / (spans * splits * rank_blocks(a.R)));
    const dim3 grid((unsigned)(spans * a.turns), rank_blocks(a.R), (unsigned)splits);
    // rows that begin between two dwords
    const uintptr_t odd = ((uintptr_t)a.x | (uintptr_t)a.stride * sizeof(TX) | (uintptr_t)a.w | (uintptr_t)a.K * sizeof(TW)) & 3;
#define PWLQ_FIRST(RT, SPAN)                                                                           \
    (!vec ? k_adapter_first<TX, TW, RT, SPAN, false, false><<<grid, 256, 0, stream>>>(a)               \
     : odd && sizeof(TX) < 4 ? k_adapter_first<TX, TW, RT, SPAN, true, (sizeof(TX) < 4)><<<grid, 256, 0, stream>>>(a) \
          : k_adapter_first<TX, TW, RT, SPAN, true, false><<<grid, 256, 0, stream>>>(a))
#define PWLQ_FIRST_SPAN(SPAN)                                                                   \
    (rank_tiles(a.R) == 1 ? PWLQ_FIRST(1, SPAN) : rank_tiles(a.R) == 2 ? PWLQ_FIRST(2, SPAN) : PWLQ_FIRST(4, SPAN))
    if (collect) PWLQ_FIRST_SPAN(kCollected);
    else PWLQ_FIRST_SPAN(kRows);
#undef PWLQ_FIRST_SPAN
#undef PWLQ_FIRST
}

void first(const FirstArgs &a, int x_type, int w_type, bool vec, hipStream_t stream)
{
    if (w_type == PWLQ_F32) x_type == PWLQ_I8 ? first_as<int8_t, float>(a, vec, stream) : first_as<float, float>(a, vec, stream);
    else if (w_type == PWLQ_BF16) x_type == PWLQ_I8 ? first_as<int8_t, bf16>(a, vec, stream) : first_as<bf16, bf16>(a, vec, stream);
    else x_type == PWLQ_I8 ? first_as<int8_t, f16>(a, vec, stream) : first_as<f16, f16>(a, vec, stream);
}


// Whether the second product does each row by itself, reading its adapter for it alone.  Both products of 4096 x 4096, 16 ranks, in us,
// by tiles -> by rows, adapters alternating: 32 rows of 8 adapters 13.5 -> 9.3, 128 rows 14.6 -> 10.5, 256 rows 14.2 -> 12.7, 384 rows
// 15.4 -> 15.7; of 32 adapters 256 rows 24.0 -> 17.1; of one adapter 128 rows 9.3 both ways, 384 rows 9.8 -> 13.7; of 8 adapters of 64
// ranks 128 rows 18.1 -> 17.0, 256 rows 19.4 -> 21.2.
bool by_rows(int64_t rows, int R, int adapters)
{
    return rows <= (adapters > 1 ? 256 : 64) && rows * ((R + 15) / 16 * 16) <= 8192;
}

template <typename TW, typename TB> void second_as(SecondArgs a, bool vec, hipStream_t stream)
{
    if (by_rows(a.rows, a.R, a.adapters)) {
        const dim3 grid((unsigned)((a.C + 511) / 512), (unsigned)a.rows);
        const int base_type = std::is_same<TB, float>::value ? PWLQ_F32 : -1;
        if (vec) k_adapter_second_row<TW, true><<<grid, 256, 0, stream>>>(a, base_type);
        else k_adapter_second_row<TW, false><<<grid, 256, 0, stream>>>(a, base_type);
        return;
    }
    const int64_t tiles = (a.rows + kSecondRows - 1) / kSecondRows, columns = (a.C + 127) / 128;
    const int waves = (int)std::min<int64_t>(columns, 4);
    const bool collect = collected(a.rows, a.R, a.adapters);
    // As many workgroups as are resident walk at once.  Of collected ones some have a second tile: with a binary32 base half as many
    // again take 25.8 us for 4096 rows where these take 28.0; with a base of 16 bits 21.9 and 20.1.
    a.walks = (int)std::min<int64_t>((columns + waves - 1) / waves, ((collect && sizeof(TB) == 4 ? 768 : 512) + tiles - 1) / tiles);
    const size_t lds = sizeof(float) * kSecondRows * second_pitch(a.R);
    if (collect) {
        const int64_t spans = (a.rows + kCollected - 1) / kCollected;
        a.turns = turns(std::min<int64_t>(a.rows, kCollected), kSecondRows, a.adapters, true, 512 / (spans * a.walks));
        const unsigned grid = (unsigned)(spans * a.turns * a.walks);
        if (vec) k_adapter_second_collected<TW, TB, true><<<grid, 64 * waves, lds, stream>>>(a);
        else k_adapter_second_collected<TW, TB, false><<<grid, 64 * waves, lds, stream>>>(a);
        return;
    }
    const unsigned grid = (unsigned)(tiles * a.walks);
    if (vec) k_adapter_second<TW, TB, true><<<grid, 64 * waves, lds, stream>>>(a);
    else k_adapter_second<TW, TB, false><<<grid, 64 * waves, lds, stream>>>(a);
}

void second(SecondArgs a, int w_type, int base_type, bool vec, hipStream_t stream)
{
    a.has_base = a.base != nullptr;
    if (!a.base) {
        a.base = a.w;
        a.base_stride = 0;
        base_type = w_type;
    }
    if (w_type == PWLQ_F32) second_as<float, float>(a, vec, stream);
    else if (w_type == PWLQ_BF16) base_type == PWLQ_F32 ? second_as<bf16, float>(a, vec, stream) : second_as<bf16, bf16>(a, vec, stream);
    else base_type == PWLQ_F32 ? second_as<f16, float>(a, vec, stream) : second_as<f16, f16>(a, vec, stream);
}

template <typename TX, typename TY> void outer_as(const OuterArgs &up, const OuterArgs &down, int splits, bool vec, hipStream_t stream)
{
    const dim3 grid((unsigned)(up.column_tiles * up.rank_blocks + down.column_tiles * down.rank_blocks), splits, up.slots);
#define PWLQ_OUTER(RT)                                                                          \
    do {                                                                                        \
        if (vec) k_adapter_outer<TX, TY, RT, true><<<grid, 256, 0, stream>>>(up, down);         \
        else k_adapter_outer<TX, TY, RT, false><<<grid, 256, 0, stream>>>(up, down);            \
    } while (0)
    if (up.R <= 16) PWLQ_OUTER(1);
    else PWLQ_OUTER(2);
#undef PWLQ_OUTER
}

void outer(const OuterArgs &up, const OuterArgs &down, int splits, int x_type, int w_type, bool vec, hipStream_t stream)
{
    if (w_type == PWLQ_F32) x_type == PWLQ_I8 ? outer_as<int8_t, float>(up, down, splits, vec, stream) : outer_as<float, float>(up, down, splits, vec, stream);
    else if (w_type == PWLQ_BF16) x_type == PWLQ_I8 ? outer_as<int8_t, bf16>(up, down, splits, vec, stream) : outer_as<bf16, bf16>(up, down, splits, vec, stream);
    else x_type == PWLQ_I8 ? outer_as<int8_t, f16>(up, down, splits, vec, stream) : outer_as<f16, f16>(up, down, splits, vec, stream);
}

// Whether rows go through one launch: few rounds of a wavefront's ranks and columns, and one workgroup to a CU, or few rows.  Against two
// launches, bfloat16, in us, 8 adapters: 1 row of 4096 x 4096 with 16 ranks 5.7 and 7.3, 16 rows 6.0 and 9.4, 32 rows 6.3 and 9.4, 48 rows
// 10.4 and 9.4; 8 rows with 32 ranks 9.1 and 10.3, with 48 11.8 and 11.9, with 64 14.9 and 12.8; 8 rows of 11008 x 4096 with 16 ranks
// 11.0 and 13.1, with 32 19.3 and 14.2; 4096 x 11008 with 16 ranks 8 rows 6.2 and 8.8, 12 rows 7.1 and 9.2, 24 rows 11.4 and 9.5.
// In binary32, whose rounds are of 2048 columns, the rule is the same: 1 row of 4096 x 4096 with 16 ranks 6.6 and 8.2, 32 rows 7.3 and
// 10.0; 8 rows with 32 ranks 13.4 and 12.0, with 48 18.3 and 14.9; of 2048 x 4096 with 48 10.4 and 13.9; of 8192 x 4096 with 16 12.8 and 11.9.
constexpr int64_t kTokenRows = 12;
bool few_ranks(int64_t K, int R) { return (R + 15) / 16 * ((K + 4095) / 4096) <= kTokenRanks / 16; }
bool by_token(int64_t T, int64_t K, int64_t N, int R)
{
    return few_ranks(K, R) && (T <= kTokenRows || T * ((N + kTokenColumns - 1) / kTokenColumns) <= 256);
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
    const bool vec = a.K >= 8 && a.N >= 8, packed = a.x.type == PWLQ_I8;
    if (a.weight_type == PWLQ_F32) packed ? token_as<int8_t, float>(t, a.T, vec, stream) : token_as<float, float>(t, a.T, vec, stream);
    else if (a.weight_type == PWLQ_BF16) packed ? token_as<int8_t, bf16>(t, a.T, vec, stream) : token_as<bf16, bf16>(t, a.T, vec, stream);
    else packed ? token_as<int8_t, f16>(t, a.T, vec, stream) : token_as<f16, f16>(t, a.T, vec, stream);
}

} // namespace

size_t adapter_workspace(int64_t T, int64_t K, int R)
{
    if (T <= kTokenRows && few_ranks(K, R)) return 0;
    const int splits = first_splits(T, K, R);
    return splits > 1 ? (size_t)splits * (size_t)T * (size_t)R * sizeof(float) : 0;
}

void adapter_forward(const pwlq_adapter_args &a, void *workspace, hipStream_t stream)
{
    if (by_token(a.T, a.K, a.N, a.R)) {
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
    first(f, a.x.type, a.weight_type, a.K >= 8, stream);
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
    second(s, a.weight_type, a.base.type, a.N >= 8, stream);
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
    first(f, a.dy.type, a.weight_type, a.N >= 8, stream);
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
    second(s, a.weight_type, a.dx_base.type,
           a.K >= 8, stream);
    OuterArgs up = {}, down = {};
    up.rows = down.rows = a.T;
    up.span = down.span = outer_span(a.T, a.K, a.N, a.R, a.adapters);
    up.ids = down.ids = a.ids;
    up.R = down.R = a.R;
    up.adapters = down.adapters = a.adapters;
    up.rank_blocks = down.rank_blocks = outer_blocks(a.R);
    up.slots = down.slots = outer_slots(a.T, a.K, a.N, a.R, a.adapters);
    up.h = a.h;
    up.x = a.dy.data;
    up.stride = a.dy.stride;
    up.C = a.N;
    up.column_tiles = (int)((a.N + 127) / 128);
    down.h = space.dh;
    down.x = a.x.data;
    down.stride = a.x.stride;
    down.step = a.x.step;
    down.C = a.K;
    down.column_tiles = (int)((a.K + 127) / 128);
    const bool join = space.splits > 1;
    up.out = join ? space.up : a.d_up;
    down.out = join ? space.down : a.d_down;
    up.present = down.present = join ? space.present : nullptr;
    up.flags = true;
    outer(up, down, space.splits, a.x.type, a.weight_type,
          a.K >= 8 && a.N >= 8, stream);
    if (!join) return;
    JoinArgs j = {};
    j.part[0] = space.down;
    j.part[1] = space.up;
    j.present = space.present;
    j.out[0] = a.d_down;
    j.out[1] = a.d_up;
    j.each[0] = a.R * a.K;
    j.each[1] = a.R * a.N;
    j.splits = space.splits;
    j.adapters = a.adapters;
    const int64_t most = std::max(j.each[0], j.each[1]);
    const dim3 grid((unsigned)std::min<int64_t>((most + 255) / 256, 1 << 16), a.adapters, 2);
    k_adapter_join<<<grid, 256, 0, stream>>>(j);
}

} // namespace pwlq_block
