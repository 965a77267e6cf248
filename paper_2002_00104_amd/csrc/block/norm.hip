// k_norm_block: the norm after a block, its gate and residual scale, the residual sum, and the norm before the next block.
// k_norm_backward, k_column_sums: its gradients.
//
//   v = f post a, a = 1/sqrt(mean f^2 + eps);  x' = x + alpha gate v;  u = x' pre b, b = 1/sqrt(mean x'^2 + eps)
// Backward, with xh = x' b, fh = f a and means over a row:
//   dx   = dx' + b (pre du - xh mean(pre du xh)),   d_pre  = sum over rows of du xh
//   dv   = alpha gate dx,                           d_gate = sum over its rows of alpha v dx
//   df   = a (post dv - fh mean(post dv fh)),       d_post = sum over rows of dv fh
// The forward pass is bound by memory: a workgroup holds a row in registers and reads each of its values once, the next row's on their
// way meanwhile.  4096 x 4096, f in bfloat16, the residual stream in binary32, codes out: 36 us, 185 MB, 5.1 TB/s; all in bfloat16 24 us,
// the norm alone 13 (replayed, inputs partly in the last-level cache); 8 rows of bfloat16 4.0 us, a launch and a row's chain of three
// reductions.
#include <algorithm>

#include "launch.h"
#include "rows.h"

#pragma clang fp contract(fast)

namespace pwlq_block {
namespace {

// Wavefronts that walk the rows at once, as many as are resident: sixteen to a CU (4096 x 4096 36.8 us; 24 43.8), and for the backward
// pass, which keeps more of a row and the columns' sums in registers, eight.
constexpr int64_t kForwardWaves = 256 * 16, kBackwardWaves = 256 * 8;

inline int threads_for(int64_t cols, int E) { return (int)((cols + 64 * E - 1) / (64 * E) * 64); }

template <typename TF, typename TX, int E, Share S, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_block(pwlq_norm_args a)
{
    __shared__ float slots[2][2][16];
    __shared__ uint32_t top[2][16];
    const int threads = blockDim.x, thread = threadIdx.x, D = (int)a.D;
    const float inv = 1.0f / (float)D;
    const int64_t per_gate = a.gate ? a.T / a.gate_rows : 1;
    Row<float, E, S> pre, post;
    Row<TF, E, S> f, gate;
    Row<TX, E, S> x;
    pre.load(a.pre_weight, Place{D, threads, thread});
    if (a.post_weight) post.load(a.post_weight, Place{D, threads, thread});
    auto load = [&](int64_t row) {
        x.load((const TX *)a.x.data + row * a.x.stride, Place{D, threads, thread});
        if (a.f.data) f.load((const TF *)a.f.data + row * a.f.stride, Place{D, threads, thread});
        if (a.gate) gate.load((const TF *)a.gate + row / per_gate * a.D, Place{D, threads, thread});
    };
    load(blockIdx.x);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1) {
        float v[E], g[E], w[E];
        x.get(v, Place{D, threads, thread});
        if (a.f.data) f.get(g, Place{D, threads, thread});
        if (a.gate) gate.get(w, Place{D, threads, thread});
        load(min(row + gridDim.x, a.T - 1));           // the next row, while this one is worked on
        loads_first();
        if (a.f.data) {
            float scale = a.alpha;
            if (a.post_weight) {
                float s = 0.0f, p[E];
#pragma unroll
                for (int i = 0; i < E; ++i) s += g[i] * g[i];
                scale *= 1.0f / sqrtf(block_sum(s, slots[turn][0], threads) * inv + a.eps);
                post.get(p, Place{D, threads, thread});
#pragma unroll
                for (int i = 0; i < E; ++i) g[i] *= p[i];
            }
            if (a.gate) {
#pragma unroll
                for (int i = 0; i < E; ++i) g[i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] += scale * g[i];
            store_row<TX, E, S>((TX *)a.x_out.data + row * a.x_out.stride, Place{D, threads, thread}, v);
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) s += v[i] * v[i];
        const float b = 1.0f / sqrtf(block_sum(s, slots[turn][1], threads) * inv + a.eps);
        pre.get(w, Place{D, threads, thread});
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = v[i] * b * w[i];
        if (a.u.type == PWLQ_I8) {
            const Step q = step_of(block_max(largest(v), top[turn], threads));
            store_codes<E, S>((int8_t *)a.u.data + row * a.u.stride, Place{D, threads, thread}, v, q.factor);
            if (thread == 0) a.u.step[row] = q.step;
        } else {
            store_row<TF, E, S>((TF *)a.u.data + row * a.u.stride, Place{D, threads, thread}, v);
        }
    }
}

// Partial sums of the parameters' gradients: walk w takes the rows [w span, (w + 1) span) and keeps a sum per column in
// registers; the next launch adds the walks' sums in order, so a gradient does not depend on timing.  Rows of up to 512 columns
// take a wavefront each, and the four walks of a workgroup first add theirs up in LDS.  A gate of several rows changes inside a
// walk.  A gate row whose rows all lie in it is written to d_gate; else the sums of walk w for gate row g are partial row w + g,
// one of its own for each pair, since from a pair to the next one of the two grows.
struct NormPartials {
    float *pre, *post, *gate;      // [workgroups, D], [workgroups, D], [workgroups * walks + gate_rows, D]
    int64_t span;
    int walks;                     // of a workgroup
};
constexpr int kWalks = 4, kWalkColumns = 512;

__device__ inline float *gate_sums(const pwlq_norm_backward_args &a, const NormPartials &part, int64_t walk, int64_t g, int64_t per,
                                   int64_t first, int64_t last)
{
    return (g * per >= first && (g + 1) * per <= last ? a.d_gate + g * a.D : part.gate + (walk + g) * a.D);
}

// Bound by memory: 4096 x 4096 of bfloat16 from 8-bit x and f 42 us for 168 MB of rows and 25 MB of partial sums (512 walks, a row for each of
// three gradients), 4.6 TB/s, and 6.7 to read those again; 515 x 1155 of binary32 10.6 and 4.1.  Some 25 vector instructions an element
// would take 11 us by themselves and are in the way only where wavefronts wait for each other at the two barriers of a row, so a
// row's factors are joined before they meet its elements: steps of 8 bits with the norms' factors, alpha and the gate with the post
// weight.  Both the gate's and the post weight's gradients are column factors times sum dx fh over the rows of one gate row, the only sum
// kept for them; where all rows have one gate row that sum could be stored once instead of twice.
template <typename TF, typename TX, bool KEPT, int E, Share S, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_backward(pwlq_norm_backward_args a, NormPartials part)
{
    typedef typename std::conditional<KEPT, int8_t, TF>::type SF;
    typedef typename std::conditional<KEPT, int8_t, TX>::type SX;
    __shared__ float2 slots[2][2][16];
    // a walk's threads: the whole workgroup, or one of its wavefronts
    const int threads = part.walks == 1 ? blockDim.x : 64, thread = part.walks == 1 ? threadIdx.x : threadIdx.x & 63, D = (int)a.D;
    const int64_t walk = (int64_t)blockIdx.x * part.walks + (part.walks == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    const float inv = 1.0f / (float)D;
    const int64_t per_gate = a.gate ? a.T / a.gate_rows : a.T;
    const int64_t first = walk * part.span, last = min(first + part.span, a.T);
    float pre[E], back[E], sum_pre[E], sum_post[E], sum_f[E];      // back: alpha gate post
#pragma unroll
    for (int i = 0; i < E; ++i) sum_pre[i] = sum_post[i] = sum_f[i] = 0.0f;
    Row<TF, E, S> du_row;
    Row<TX, E, S> dx_row;
    Row<SX, E, S> x_row;
    Row<SF, E, S> f_row;
    float x_step = 1.0f, f_step = 1.0f;
    auto load = [&](int64_t row) {
        x_row.load((const SX *)a.x_out.data + row * a.x_out.stride, Place{D, threads, thread});
        if (a.du.data) du_row.load((const TF *)a.du.data + row * a.du.stride, Place{D, threads, thread});
        if (a.dx_out.data) dx_row.load((const TX *)a.dx_out.data + row * a.dx_out.stride, Place{D, threads, thread});
        if (a.f.data) f_row.load((const SF *)a.f.data + row * a.f.stride, Place{D, threads, thread});
        if (KEPT) x_step = a.x_out.step[row];
        if (KEPT && a.f.data) f_step = a.f.step[row];
    };
    // alpha gate into g, post into p
    constexpr bool kHold = E == 8;                     // post stays in registers where there is room
    Row<float, E, S> post;
    Row<TF, E, S> gate;
    auto factors = [&](float (&g)[E], float (&p)[E]) {
#pragma unroll
        for (int i = 0; i < E; ++i) g[i] = p[i] = 1.0f;
        if (a.post_weight) {
            if (!kHold) post.load(a.post_weight, Place{D, threads, thread});
            post.get(p, Place{D, threads, thread});
        }
        if (a.gate) gate.get(g, Place{D, threads, thread});
#pragma unroll
        for (int i = 0; i < E; ++i) g[i] *= a.alpha;
    };
    // the sums of a gate row's end
    auto settle = [&](int64_t gate_row) {
        float g[E], p[E];
        factors(g, p);
#pragma unroll
        for (int i = 0; i < E; ++i) {
            sum_post[i] += g[i] * sum_f[i];
            sum_f[i] *= a.alpha * p[i];
        }
        if (a.gate) store_row<float, E, S>(gate_sums(a, part, walk, gate_row, per_gate, first, last), Place{D, threads, thread}, sum_f);
#pragma unroll
        for (int i = 0; i < E; ++i) sum_f[i] = 0.0f;
    };
    Row<float, E, S> weight;
    weight.load(a.pre_weight, Place{D, threads, thread});
    if (kHold && a.post_weight) post.load(a.post_weight, Place{D, threads, thread});
    if (a.gate && first < last) gate.load((const TF *)a.gate + first / per_gate * a.D, Place{D, threads, thread});
    if (first < last) load(first);
    loads_first();
    weight.get(pre, Place{D, threads, thread});
    int64_t at_gate = -1;
    int turn = 0;
    for (int64_t row = first; row < last; ++row, turn ^= 1) {
        float dx[E], x[E], f[E], du[E];
        x_row.get(x, Place{D, threads, thread});
        if (a.f.data) f_row.get(f, Place{D, threads, thread});
        if (a.du.data) du_row.get(du, Place{D, threads, thread});
        if (a.dx_out.data) dx_row.get(dx, Place{D, threads, thread});
        else {
#pragma unroll
            for (int i = 0; i < E; ++i) dx[i] = 0.0f;
        }
        const float xs = x_step, fs = f_step;
        if (a.f.data && row / per_gate != at_gate) {
            if (at_gate >= 0) {
                settle(at_gate);
                if (a.gate) gate.load((const TF *)a.gate + row / per_gate * a.D, Place{D, threads, thread});
            }
            at_gate = row / per_gate;
            float p[E];
            factors(back, p);
#pragma unroll
            for (int i = 0; i < E; ++i) back[i] *= p[i];
        }
        load(min(row + 1, last - 1));                  // the next row, while this one is worked on
        loads_first();
        if (a.du.data) {
            float s = 0.0f, t = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                s += x[i] * x[i];
                t += x[i] * (pre[i] * du[i]);
            }
            block_sum2(s, t, slots[turn][0], threads);
            const float b = 1.0f / sqrtf(s * xs * xs * inv + a.eps), xb = xs * b, mean = t * xb * inv * b * xb;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                dx[i] = dx[i] + b * (pre[i] * du[i]) - mean * x[i];
                sum_pre[i] += du[i] * (x[i] * xb);
            }
        }
        store_row<TX, E, S>((TX *)a.dx.data + row * a.dx.stride, Place{D, threads, thread}, dx);
        if (!a.f.data) continue;
        if (a.post_weight) {
            float s = 0.0f, t = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                s += f[i] * f[i];
                t += f[i] * (back[i] * dx[i]);
            }
            block_sum2(s, t, slots[turn][1], threads);
            const float c = 1.0f / sqrtf(s * fs * fs * inv + a.eps), fc = fs * c, mean = t * fc * inv * c * fc;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                sum_f[i] += dx[i] * (f[i] * fc);
                dx[i] = c * (back[i] * dx[i]) - mean * f[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                sum_f[i] += dx[i] * (f[i] * fs);
                dx[i] *= back[i];
            }
        }
        store_row<TF, E, S>((TF *)a.df.data + row * a.df.stride, Place{D, threads, thread}, dx);
    }
    if (at_gate >= 0) settle(at_gate);
    if constexpr (E == 8) {
        if (part.walks > 1) {                          // the other walks' sums, in order
            __shared__ float sums[kWalks - 1][2][kWalkColumns];
            const int wave = threadIdx.x >> 6;
            if (wave) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    sums[wave - 1][0][64 * i + thread] = sum_pre[i];
                    sums[wave - 1][1][64 * i + thread] = sum_post[i];
                }
            }
            __syncthreads();
            if (wave) return;
#pragma unroll
            for (int w = 0; w < kWalks - 1; ++w)
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    sum_pre[i] += sums[w][0][64 * i + thread];
                    sum_post[i] += sums[w][1][64 * i + thread];
                }
        }
    }
    store_row<float, E, S>(part.pre + (int64_t)blockIdx.x * a.D, Place{D, threads, thread}, sum_pre);
    if (part.post) store_row<float, E, S>(part.post + (int64_t)blockIdx.x * a.D, Place{D, threads, thread}, sum_post);
}

// Sums of the partial rows, in order: of all workgroups for the norms' weights, of those that meet it for a gate row.  Sixteen
// wavefronts take a row each in turn, four loads under way.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void k_column_sums(pwlq_norm_backward_args a, NormPartials part, int workgroups, int64_t outs)
{
    __shared__ float sums[kSumWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = min((int64_t)blockIdx.x * 64 + lane, a.D - 1);
    // outputs: d_pre, d_post, the rows of d_gate
    for (int64_t out = blockIdx.y; out < outs; out += gridDim.y) {
        const float *from = out == 0 ? part.pre : part.post;
        float *to = out == 0 ? a.d_pre : a.d_post;
        int64_t first = 0, last = workgroups;
        if (out >= 2) {
            const int64_t g = out - 2, per = a.T / a.gate_rows;
            from = part.gate + g * a.D;
            to = a.d_gate + g * a.D;
            first = g * per / part.span;
            last = ((g + 1) * per - 1) / part.span + 1;
            if (last - first == 1) continue;            // written by the one workgroup
        }
        if (!to) continue;
        float s = 0.0f;
        for (int64_t w = first + wave; w < last; w += 8 * kSumWaves) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = from[min(w + j * kSumWaves, last - 1) * a.D + col];
            loads_first();
#pragma unroll
            for (int j = 0; j < 8; ++j) s += w + j * kSumWaves < last ? v[j] : 0.0f;
        }
        __syncthreads();
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && blockIdx.x * 64 + lane < a.D) {
#pragma unroll
            for (int i = 1; i < kSumWaves; ++i) s += sums[i][lane];
            to[col] = s;
        }
    }
}

__global__ void k_zero(float *a, int64_t na, float *b, int64_t nb, float *c, int64_t nc)
{
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
    for (int64_t j = i; j < na; j += step) a[j] = 0.0f;
    for (int64_t j = i; j < nb; j += step) b[j] = 0.0f;
    for (int64_t j = i; j < nc; j += step) c[j] = 0.0f;
}

// Elements of a thread, by the row's length, and the registers a kernel may have by its most threads.  The forward pass takes 8 up
// to 4096 columns and 16 beyond; the backward pass 8 up to 2048, 16 beyond (at 4096 16 of 256 threads 45.6 us, 8 of 512
// 55.5: fewer wavefronts meet at each of its two barriers a row).
// Beyond 8192 columns a workgroup has more than 512 threads, which leaves a thread 128 registers.  The forward pass spills 10 to 85 of
// them, none with whole vectors of 16 bits throughout (2048 x 16384 47.6 us, 5.6 TB/s; all in binary32 181, 3.0 TB/s); the backward
// pass, which keeps five values a column, 160 to 342: 4096 x 12288 of bfloat16 599 us and 2048 x 16384 468, 0.9 to 1.0 TB/s, where
// 4096 x 8192 takes 98, 4.1 TB/s (replayed, inputs partly in the last-level cache).
int forward_elements(int64_t D) { return D <= 4096 ? 8 : 16; }
int backward_elements(int64_t D) { return D <= 2048 ? 8 : 16; }

int backward_walks(int64_t D) { return D <= kWalkColumns ? kWalks : 1; }
// Rows of a walk: two at least, since what a walk leaves behind is read again.  Both kernels with at least 1, 2 and 3 rows, in us: 515 x 1155
// of binary32 16.4, 12.9 and 13.6, 300 x 4096 of bfloat16 19.6, 16.4 and 16.4, 1500 x 296 18.9, 14.0 and 12.9; with so few rows that they wait
// for nothing else 130 x 600 of binary32 8.3, 9.2 and 10.5, 40 x 8192 12.9, 14.1 and 16.1.
int64_t backward_span(int64_t T, int64_t D)
{
    const int64_t walks = kBackwardWaves / (threads_for(D, backward_elements(D)) / 64);
    return std::max<int64_t>((T + walks - 1) / walks, 2);
}
int64_t backward_wgs(int64_t T, int64_t D)
{
    const int64_t rows = backward_span(T, D) * backward_walks(D);
    return (T + rows - 1) / rows;
}

template <typename TF, typename TX, Share S> void norm_as(const pwlq_norm_args &a, hipStream_t stream)
{
    const int64_t wgs = kForwardWaves / (threads_for(a.D, forward_elements(a.D)) / 64);
    const unsigned grid = (unsigned)std::min(a.T, wgs);
#define PWLQ_NORM(E, THREADS) k_norm_block<TF, TX, E, S, THREADS><<<grid, threads_for(a.D, E), 0, stream>>>(a)
    if (a.D <= 4096) PWLQ_NORM(8, 512);
    else if (a.D <= 8192) PWLQ_NORM(16, 512);
    else PWLQ_NORM(16, 1024);
#undef PWLQ_NORM
}

template <typename TF, typename TX, bool KEPT, Share S>
void backward_as(const pwlq_norm_backward_args &a, const NormPartials &part, unsigned grid, hipStream_t stream)
{
    const int threads = part.walks * threads_for(a.D, backward_elements(a.D));
#define PWLQ_NORM(E, THREADS) k_norm_backward<TF, TX, KEPT, E, S, THREADS><<<grid, threads, 0, stream>>>(a, part)
    if constexpr (S != kTail)
        if (a.D <= 2048) return PWLQ_NORM(8, 256);
    if constexpr (S != kSingly) {
        if (a.D <= 8192) PWLQ_NORM(16, 512);
        else PWLQ_NORM(16, 1024);
    }
#undef PWLQ_NORM
}

} // namespace

void norm_block(const pwlq_norm_args &a, hipStream_t stream)
{
    const int tf = a.f.data ? a.f.type : a.x.type;
    // Rows of no whole vectors: a residual stream of 16 bits moves in vectors all the same (2000 x 4090 16.1 us, singly 19.4), one of
    // binary32 singly (22.6, in vectors 24.7).
#define PWLQ_AS(TF, TX)                                                                             \
    (a.D % 8 == 0                       ? norm_as<TF, TX, kWhole>(a, stream)                        \
     : sizeof(TX) == 2 && a.D >= 8      ? norm_as<TF, TX, sizeof(TX) == 2 ? kTail : kWhole>(a, stream) \
                                        : norm_as<TF, TX, kSingly>(a, stream))
    if (tf == PWLQ_F32) PWLQ_AS(float, float);
    else if (tf == PWLQ_BF16 && a.x.type == PWLQ_BF16) PWLQ_AS(bf16, bf16);
    else if (tf == PWLQ_BF16) PWLQ_AS(bf16, float);
    else if (a.x.type == PWLQ_F16) PWLQ_AS(f16, f16);
    else PWLQ_AS(f16, float);
#undef PWLQ_AS
}

// Partial rows in the workspace: d_pre's, d_post's, then d_gate's, which has one for each gate row also where those that lie within a walk
// never use theirs: with a gate for each row as many bytes as d_gate.
size_t norm_backward_workspace(int64_t T, int64_t D, int64_t gate_rows)
{
    if (!T) return 0;
    return (size_t)(backward_wgs(T, D) * (2 + backward_walks(D)) + gate_rows) * (size_t)D * sizeof(float);
}

void norm_backward(const pwlq_norm_backward_args &a, void *workspace, hipStream_t stream)
{
    if (a.T == 0) {
        const int64_t n = a.d_gate ? a.gate_rows * a.D : 0;
        k_zero<<<256, 256, 0, stream>>>(a.d_pre, a.d_pre ? a.D : 0, a.d_post, a.d_post ? a.D : 0, a.d_gate, n);
        return;
    }
    const int64_t wgs = backward_wgs(a.T, a.D);
    NormPartials part = {(float *)workspace, a.d_post ? (float *)workspace + wgs * a.D : nullptr,
                         (float *)workspace + 2 * wgs * a.D, backward_span(a.T, a.D), backward_walks(a.D)};
    const bool kept = a.x_out.type == PWLQ_I8;
    const int tx = a.dx.type, tf = a.f.data ? a.df.type : a.du.data ? a.du.type : tx;
#define PWLQ_AS(TF, TX) (kept ? PWLQ_SHARE(TF, TX, true) : PWLQ_SHARE(TF, TX, false))
    // Rows of no whole vectors move in vectors where a thread has sixteen columns (2000 x 4090 of bfloat16 with 8-bit checkpoints 37 us,
    // singly 69), singly where it has eight (4000 x 515 28.4, in vectors 28.9).
#define PWLQ_SHARE(TF, TX, KEPT)                                                                     \
    (a.D % 8 == 0    ? backward_as<TF, TX, KEPT, kWhole>(a, part, (unsigned)wgs, stream)             \
     : a.D > 2048    ? backward_as<TF, TX, KEPT, kTail>(a, part, (unsigned)wgs, stream)              \
                     : backward_as<TF, TX, KEPT, kSingly>(a, part, (unsigned)wgs, stream))
    if (tf == PWLQ_F32) PWLQ_AS(float, float);
    else if (tf == PWLQ_BF16 && tx == PWLQ_BF16) PWLQ_AS(bf16, bf16);
    else if (tf == PWLQ_BF16) PWLQ_AS(bf16, float);
    else if (tx == PWLQ_F16) PWLQ_AS(f16, f16);
    else PWLQ_AS(f16, float);
#undef PWLQ_SHARE
#undef PWLQ_AS
    // gate rows that lie within walks are written already
    const bool straddled = a.d_gate && part.span % (a.T / a.gate_rows) != 0;
    const int64_t outs = 2 + (straddled ? a.gate_rows : 0);
    const dim3 grid((unsigned)((a.D + 63) / 64), (unsigned)(outs < 4096 ? outs : 4096));
    k_column_sums<<<grid, 64 * kSumWaves, 0, stream>>>(a, part, (int)wgs, outs);
}

} // namespace pwlq_block
