// k_norm_block: the norm after a block, its gate and residual scale, the residual sum, and the norm before the next block.
// k_norm_backward, k_column_sums: its gradients.
//
//   v = f post a, a = 1/sqrt(mean f^2 + eps);  x' = x + alpha gate v;  u = x' pre b, b = 1/sqrt(mean x'^2 + eps)
// Backward, with xh = x' b, fh = f a and means over a row:
//   dx   = dx' + b (pre du - xh mean(pre du xh)),   d_pre  = sum over rows of du xh
//   dv   = alpha gate dx,                           d_gate = sum over its rows of alpha v dx
//   df   = a (post dv - fh mean(post dv fh)),       d_post = sum over rows of dv fh
// All of it is bound by memory: a workgroup holds a row in registers and reads each of its values once.
#include "launch.h"
#include "rows.h"

#pragma clang fp contract(fast)

namespace pwlq_block {
namespace {

inline int threads_for(int64_t cols, int E) { return (int)((cols + 64 * E - 1) / (64 * E) * 64); }

template <typename TF, typename TX, int E, bool VEC>
__global__ __launch_bounds__(1024) void k_norm_block(pwlq_norm_args a)
{
    __shared__ float slots[2][2][16];
    __shared__ uint32_t top[2][16];
    const int threads = blockDim.x, thread = threadIdx.x, D = (int)a.D;
    const float inv = 1.0f / (float)D;
    const int64_t per_gate = a.gate ? a.T / a.gate_rows : 1;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1) {
        float x[E], w[E];
        load_row<TX, E, VEC>((const TX *)a.x.data + row * a.x.stride, D, threads, thread, x);
        if (a.f.data) {
            float f[E];
            load_row<TF, E, VEC>((const TF *)a.f.data + row * a.f.stride, D, threads, thread, f);
            float scale = a.alpha;
            if (a.post_weight) {
                load_row<float, E, VEC>(a.post_weight, D, threads, thread, w);
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < E; ++i) s += f[i] * f[i];
                scale *= 1.0f / sqrtf(block_sum(s, slots[turn][0], threads) * inv + a.eps);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] *= w[i];
            }
            if (a.gate) {
                load_row<TF, E, VEC>((const TF *)a.gate + row / per_gate * a.D, D, threads, thread, w);
#pragma unroll
                for (int i = 0; i < E; ++i) f[i] *= w[i];
            }
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] += scale * f[i];
            store_row<TX, E, VEC>((TX *)a.x_out.data + row * a.x_out.stride, D, threads, thread, x);
        }
        load_row<float, E, VEC>(a.pre_weight, D, threads, thread, w);
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < E; ++i) s += x[i] * x[i];
        const float b = 1.0f / sqrtf(block_sum(s, slots[turn][1], threads) * inv + a.eps);
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = x[i] * b * w[i];
        if (a.u.type == PWLQ_I8) {
            const Step q = step_of(block_max(largest(x), top[turn], threads));
            store_codes<E, VEC>((int8_t *)a.u.data + row * a.u.stride, D, threads, thread, x, q.factor);
            if (thread == 0) a.u.step[row] = q.step;
        } else {
            store_row<TF, E, VEC>((TF *)a.u.data + row * a.u.stride, D, threads, thread, x);
        }
    }
}

// Partial sums of the parameters' gradients: workgroup w walks the rows [w span, (w + 1) span) and keeps a sum per column
// in registers; the next launch adds the workgroups' sums in order, so a gradient does not depend on timing.  A
// gate of several rows changes inside the walk.  A gate row whose rows all lie in it is written to d_gate; else the sums
// of workgroup w for gate row g are partial row w + g, one of its own for each pair, since from a pair to the next one of the two grows.
struct NormPartials {
    float *pre, *post, *gate;      // [workgroups, D], [workgroups, D], [workgroups + gate_rows, D]
    int64_t span;
};

__device__ inline float *gate_sums(const pwlq_norm_backward_args &a, const NormPartials &part, int64_t g, int64_t per, int64_t first, int64_t last)
{
    return (g * per >= first && (g + 1) * per <= last ? a.d_gate + g * a.D : part.gate + ((int64_t)blockIdx.x + g) * a.D);
}

template <typename TF, typename TX, bool KEPT, int E, bool VEC>
__global__ __launch_bounds__(1024) void k_norm_backward(pwlq_norm_backward_args a, NormPartials part)
{
    typedef typename std::conditional<KEPT, int8_t, TF>::type SF;
    typedef typename std::conditional<KEPT, int8_t, TX>::type SX;
    __shared__ float slots[2][4][16];
    const int threads = blockDim.x, thread = threadIdx.x, D = (int)a.D;
    const float inv = 1.0f / (float)D;
    const int64_t per_gate = a.gate ? a.T / a.gate_rows : 1;
    const int64_t first = (int64_t)blockIdx.x * part.span, last = min(first + part.span, a.T);
    float sum_pre[E], sum_post[E], sum_gate[E], gate[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        sum_pre[i] = sum_post[i] = sum_gate[i] = 0.0f;
        gate[i] = 1.0f;
    }
    int64_t at_gate = -1;
    int turn = 0;
    for (int64_t row = first; row < last; ++row, turn ^= 1) {
        float dx[E], x[E], f[E], du[E], w[E];
        load_row<SX, E, VEC>((const SX *)a.x_out.data + row * a.x_out.stride, D, threads, thread, x);
        if (a.du.data) load_row<TF, E, VEC>((const TF *)a.du.data + row * a.du.stride, D, threads, thread, du);
        if (a.dx_out.data) load_row<TX, E, VEC>((const TX *)a.dx_out.data + row * a.dx_out.stride, D, threads, thread, dx);
        if (a.f.data) load_row<SF, E, VEC>((const SF *)a.f.data + row * a.f.stride, D, threads, thread, f);
        if (a.gate && row / per_gate != at_gate) {
            if (at_gate >= 0) {
                store_row<float, E, VEC>(gate_sums(a, part, at_gate, per_gate, first, last), D, threads, thread, sum_gate);
#pragma unroll
                for (int i = 0; i < E; ++i) sum_gate[i] = 0.0f;
            }
            at_gate = row / per_gate;
            load_row<TF, E, VEC>((const TF *)a.gate + at_gate * a.D, D, threads, thread, gate);
        }
        if (!a.dx_out.data) {
#pragma unroll
            for (int i = 0; i < E; ++i) dx[i] = 0.0f;
        }
        if (a.du.data) {
            if constexpr (KEPT) {
                const float step = a.x_out.step[row];
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] *= step;
            }
            load_row<float, E, VEC>(a.pre_weight, D, threads, thread, w);
            float s = 0.0f, t = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                s += x[i] * x[i];
                t += x[i] * (w[i] * du[i]);
            }
            s = block_sum(s, slots[turn][0], threads);
            t = block_sum(t, slots[turn][1], threads);
            const float b = 1.0f / sqrtf(s * inv + a.eps), mean = t * inv * b * b;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                dx[i] += b * (w[i] * du[i] - x[i] * mean);
                sum_pre[i] += du[i] * (x[i] * b);
            }
        }
        store_row<TX, E, VEC>((TX *)a.dx.data + row * a.dx.stride, D, threads, thread, dx);
        if (!a.f.data) continue;
        if constexpr (KEPT) {
            const float step = a.f.step[row];
#pragma unroll
            for (int i = 0; i < E; ++i) f[i] *= step;
        }
        // dx becomes dv / gate, then dv
#pragma unroll
        for (int i = 0; i < E; ++i) dx[i] *= a.alpha;
        if (a.post_weight) {
            load_row<float, E, VEC>(a.post_weight, D, threads, thread, w);
            float s = 0.0f, t = 0.0f;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                s += f[i] * f[i];
                t += f[i] * (w[i] * (gate[i] * dx[i]));
            }
            s = block_sum(s, slots[turn][2], threads);
            t = block_sum(t, slots[turn][3], threads);
            const float c = 1.0f / sqrtf(s * inv + a.eps), mean = t * inv * c * c;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float dv = gate[i] * dx[i], fh = f[i] * c;
                sum_gate[i] += dx[i] * (fh * w[i]);
                sum_post[i] += dv * fh;
                dx[i] = c * (w[i] * dv - f[i] * mean);
            }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                sum_gate[i] += dx[i] * f[i];
                dx[i] *= gate[i];
            }
        }
        store_row<TF, E, VEC>((TF *)a.df.data + row * a.df.stride, D, threads, thread, dx);
    }
    store_row<float, E, VEC>(part.pre + (int64_t)blockIdx.x * a.D, D, threads, thread, sum_pre);
    if (part.post) store_row<float, E, VEC>(part.post + (int64_t)blockIdx.x * a.D, D, threads, thread, sum_post);
    if (at_gate >= 0) store_row<float, E, VEC>(gate_sums(a, part, at_gate, per_gate, first, last), D, threads, thread, sum_gate);
}

// Sums of the partial rows: of all workgroups for the norms' weights, of those that meet it for a gate row.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(64 * kSumWaves) void k_column_sums(pwlq_norm_backward_args a, NormPartials part, int workgroups)
{
    __shared__ float sums[kSumWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    // outputs: d_pre, d_post, the rows of d_gate
    for (int64_t out = blockIdx.y; out < 2 + (a.d_gate ? a.gate_rows : 0); out += gridDim.y) {
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
        if (col < a.D)
            for (int64_t w = first + wave; w < last; w += kSumWaves) s += from[w * a.D + col];
        __syncthreads();
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && col < a.D) {
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

// Workgroups of the backward pass, each with sums of its own.
constexpr int64_t kBackwardWgs = 512;
int64_t backward_span(int64_t T) { return (T + kBackwardWgs - 1) / kBackwardWgs; }

template <typename TF, typename TX> void norm_as(const pwlq_norm_args &a, bool vec, hipStream_t stream)
{
    const unsigned grid = row_grid(a.T);
#define PWLQ_NORM(E)                                                                                    \
    do {                                                                                                \
        if (vec) k_norm_block<TF, TX, E, true><<<grid, threads_for(a.D, E), 0, stream>>>(a);            \
        else k_norm_block<TF, TX, E, false><<<grid, threads_for(a.D, E), 0, stream>>>(a);               \
    } while (0)
    if (a.D <= 8192) PWLQ_NORM(8);
    else PWLQ_NORM(16);
#undef PWLQ_NORM
}

template <typename TF, typename TX, bool KEPT>
void backward_as(const pwlq_norm_backward_args &a, const NormPartials &part, unsigned grid, bool vec, hipStream_t stream)
{
#define PWLQ_NORM(E)                                                                                            \
    do {                                                                                                        \
        if (vec) k_norm_backward<TF, TX, KEPT, E, true><<<grid, threads_for(a.D, E), 0, stream>>>(a, part);     \
        else k_norm_backward<TF, TX, KEPT, E, false><<<grid, threads_for(a.D, E), 0, stream>>>(a, part);        \
    } while (0)
    if (a.D <= 8192) PWLQ_NORM(8);
    else PWLQ_NORM(16);
#undef PWLQ_NORM
}

} // namespace

void norm_block(const pwlq_norm_args &a, hipStream_t stream)
{
    const bool vec = a.D % 8 == 0 && vectors(a.x, a.T) && vectors(a.f, a.T) && vectors(a.x_out, a.T) && vectors(a.u, a.T) &&
                     aligned16(a.post_weight) && aligned16(a.pre_weight) && aligned16(a.gate);
    const int tf = a.f.data ? a.f.type : a.x.type;
    if (tf == PWLQ_F32) norm_as<float, float>(a, vec, stream);
    else if (tf == PWLQ_BF16 && a.x.type == PWLQ_BF16) norm_as<bf16, bf16>(a, vec, stream);
    else if (tf == PWLQ_BF16) norm_as<bf16, float>(a, vec, stream);
    else if (a.x.type == PWLQ_F16) norm_as<f16, f16>(a, vec, stream);
    else norm_as<f16, float>(a, vec, stream);
}

// Partial rows in the workspace: d_pre's, d_post's, then d_gate's.
size_t norm_backward_workspace(int64_t T, int64_t D, int64_t gate_rows)
{
    if (!T) return 0;
    const int64_t wgs = (T + backward_span(T) - 1) / backward_span(T);
    return (size_t)(3 * wgs + gate_rows) * (size_t)D * sizeof(float);
}

void norm_backward(const pwlq_norm_backward_args &a, void *workspace, hipStream_t stream)
{
    if (a.T == 0) {
        const int64_t n = a.d_gate ? a.gate_rows * a.D : 0;
        k_zero<<<256, 256, 0, stream>>>(a.d_pre, a.d_pre ? a.D : 0, a.d_post, a.d_post ? a.D : 0, a.d_gate, n);
        return;
    }
    const int64_t span = backward_span(a.T), wgs = (a.T + span - 1) / span;
    NormPartials part = {(float *)workspace, a.d_post ? (float *)workspace + wgs * a.D : nullptr,
                         (float *)workspace + 2 * wgs * a.D, span};
    const bool vec = a.D % 8 == 0 && vectors(a.du, a.T) && vectors(a.dx_out, a.T) && vectors(a.x_out, a.T) &&
                     vectors(a.f, a.T) && vectors(a.dx, a.T) && vectors(a.df, a.T) && aligned16(a.post_weight) &&
                     aligned16(a.pre_weight) && aligned16(a.gate) && aligned16(a.d_gate);
    const bool kept = a.x_out.type == PWLQ_I8;
    const int tx = a.dx.type, tf = a.f.data ? a.df.type : a.du.data ? a.du.type : tx;
#define PWLQ_AS(TF, TX)                                                                              \
    (kept ? backward_as<TF, TX, true>(a, part, (unsigned)wgs, vec, stream)                           \
          : backward_as<TF, TX, false>(a, part, (unsigned)wgs, vec, stream))
    if (tf == PWLQ_F32) PWLQ_AS(float, float);
    else if (tf == PWLQ_BF16 && tx == PWLQ_BF16) PWLQ_AS(bf16, bf16);
    else if (tf == PWLQ_BF16) PWLQ_AS(bf16, float);
    else if (tx == PWLQ_F16) PWLQ_AS(f16, f16);
    else PWLQ_AS(f16, float);
#undef PWLQ_AS
    const int64_t outs = 2 + (a.d_gate ? a.gate_rows : 0);
    const dim3 grid((unsigned)((a.D + 63) / 64), (unsigned)(outs < 4096 ? outs : 4096));
    k_column_sums<<<grid, 64 * kSumWaves, 0, stream>>>(a, part, (int)wgs);
}

} // namespace pwlq_block
