// The entry points of pwlq_block.h: checks of their arguments, then the launches of launch.h.
#pragma once

#include "launch.h"

namespace {

// Grids of all launches stay below 2^32 threads a dimension.  Most have the adapters' collected tiles: 24 workgroups of 256 threads for
// each 256 rows, 1.6e9 threads, once the rows alone fill the chip; columns add none to that.
constexpr int64_t kMostRows = 1LL << 26;

constexpr int64_t kMostStride = 1LL << 20;     // 256 rows of binary32 stay below 2 GiB
bool float_type(int type) { return type == PWLQ_F32 || type == PWLQ_BF16 || type == PWLQ_F16; }

// Rows of `cols` columns that have to be there: type (codes only where `codes`), step, stride, alignment to their own elements.
int check_rows(const char *name, const pwlq_rows &r, int64_t cols, bool codes, bool row_factors = false)
{
    if (!r.data) return fail(PWLQ_ENULL, "%s is NULL", name);
    if (!float_type(r.type) && !(codes && r.type == PWLQ_I8)) return fail(PWLQ_EINVAL, "%s has type %d, not taken here", name, r.type);
    if (r.type == PWLQ_I8 && !r.step) return fail(PWLQ_ENULL, "%s is of 8 bits and has no steps", name);
    if (r.type != PWLQ_I8 && r.step && !row_factors) return fail(PWLQ_EINVAL, "%s is not of 8 bits and has steps", name);
    if (r.stride < cols) return fail(PWLQ_EINVAL, "%s: a stride of %lld for %lld columns", name, (long long)r.stride, (long long)cols);
    if ((uintptr_t)r.data % (uintptr_t)pwlq_block::type_size(r.type) != 0 || (uintptr_t)r.step % 4 != 0)
        return fail(PWLQ_EINVAL, "%s is not aligned to its elements", name);
    return PWLQ_OK;
}

int check_sizes(int64_t T, int64_t cols, int64_t most)
{
    if (T < 0 || T > kMostRows) return fail(PWLQ_EINVAL, "T=%lld outside [0,%lld]", (long long)T, (long long)kMostRows);
    if (cols < 1 || cols > most) return fail(PWLQ_EINVAL, "%lld columns: 1 to %lld are taken", (long long)cols, (long long)most);
    return PWLQ_OK;
}

int check_room(const void *workspace, size_t bytes, size_t need)
{
    if (!need) return PWLQ_OK;
    if (!workspace) return fail(PWLQ_EWORKSPACE, "workspace is NULL (%zu bytes needed)", need);
    if (((uintptr_t)workspace & 255) != 0) return fail(PWLQ_EWORKSPACE, "workspace is not 256-byte aligned");
    if (bytes < need) return fail(PWLQ_EWORKSPACE, "workspace holds %zu bytes, %zu needed", bytes, need);
    return PWLQ_OK;
}

int check_gate(const void *gate, int64_t gate_rows, int64_t T)
{
    if (gate && (gate_rows < 1 || T % gate_rows != 0))
        return fail(PWLQ_EINVAL, "gate_rows=%lld does not divide T=%lld", (long long)gate_rows, (long long)T);
    return PWLQ_OK;
}

int check_adapter(int64_t T, int64_t K, int64_t N, int R, int adapters, int type, const void *down, const void *up, const int32_t *ids,
                  const float *scale)
{
    if (int rc = check_sizes(T, K, 1 << 20)) return rc;
    if (int rc = check_sizes(T, N, 1 << 20)) return rc;
    if (R < 1 || R > 256) return fail(PWLQ_EINVAL, "R=%d outside [1,256]", R);
    if (adapters < 1 || adapters > 65535) return fail(PWLQ_EINVAL, "adapters=%d outside [1,65535]", adapters);
    if (!float_type(type)) return fail(PWLQ_EINVAL, "weight_type=%d is none of the float types", type);
    // rows and adapters are addressed within tiles by 32 bits
    const int64_t most = (1LL << 31) / pwlq_block::type_size(type);
    if (R * K >= most || R * N >= most) return fail(PWLQ_EINVAL, "an adapter of 2 GiB or more");
    if (!down || !up || !scale || (T && !ids)) return fail(PWLQ_ENULL, "an input pointer is NULL");
    if (((uintptr_t)down | (uintptr_t)up) % (uintptr_t)pwlq_block::type_size(type) != 0)
        return fail(PWLQ_EINVAL, "down or up is not aligned to its elements");
    return PWLQ_OK;
}

int check_columns(const char *name, const pwlq_rows &r, int64_t cols, int weight_type, bool codes = false, bool row_factors = false)
{
    if (int rc = check_rows(name, r, cols, codes, row_factors)) return rc;
    if (r.stride > kMostStride) return fail(PWLQ_EINVAL, "%s: a stride of %lld, over %lld", name, (long long)r.stride, (long long)kMostStride);
    if (r.type != weight_type && r.type != (codes ? PWLQ_I8 : PWLQ_F32))
        return fail(PWLQ_EINVAL, "%s has type %d beside weights of type %d", name, r.type, weight_type);
    return PWLQ_OK;
}

} // namespace

extern "C" {

int pwlq_pack_rows(const pwlq_rows *x, int64_t T, int64_t K, int8_t *codes, float *step, void *stream)
{
    if (!x) return fail(PWLQ_ENULL, "x is NULL");
    if (int rc = check_sizes(T, K, 65536)) return rc;
    if (T == 0) return PWLQ_OK;
    if (int rc = check_rows("x", *x, K, false)) return rc;
    if (!codes || !step) return fail(PWLQ_ENULL, "an output pointer is NULL");
    pwlq_block::pack_rows(*x, T, (int)K, codes, step, (hipStream_t)stream);
    return launch_status("pack launch");
}

int pwlq_unpack_rows(const int8_t *codes, const float *step, int64_t T, int64_t K, const pwlq_rows *out, void *stream)
{
    if (!out) return fail(PWLQ_ENULL, "out is NULL");
    if (int rc = check_sizes(T, K, 65536)) return rc;
    if (T == 0) return PWLQ_OK;
    if (int rc = check_rows("out", *out, K, false)) return rc;
    if (!codes || !step) return fail(PWLQ_ENULL, "an input pointer is NULL");
    pwlq_block::unpack_rows(codes, step, T, (int)K, *out, (hipStream_t)stream);
    return launch_status("unpack launch");
}

int pwlq_norm_block(const pwlq_norm_args *a, void *stream)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_sizes(a->T, a->D, 16384)) return rc;
    if (int rc = check_gate(a->gate, a->gate_rows, a->T)) return rc;
    if (a->T == 0) return PWLQ_OK;
    if (int rc = check_rows("x", a->x, a->D, false)) return rc;
    if (!a->pre_weight) return fail(PWLQ_ENULL, "pre_weight is NULL");
    int type = a->x.type;
    if (a->f.data) {
        if (int rc = check_rows("f", a->f, a->D, false)) return rc;
        if (int rc = check_rows("x_out", a->x_out, a->D, false)) return rc;
        type = a->f.type;
        if (a->x_out.type != a->x.type || (a->x.type != type && a->x.type != PWLQ_F32))
            return fail(PWLQ_EINVAL, "x and x_out have one type, f's or PWLQ_F32");
    } else if (a->post_weight || a->gate) {
        return fail(PWLQ_EINVAL, "post_weight and gate go with f");
    }
    if (int rc = check_rows("u", a->u, a->D, true)) return rc;
    if (a->u.type != type && a->u.type != PWLQ_I8) return fail(PWLQ_EINVAL, "u has type %d, not %d or PWLQ_I8", a->u.type, type);
    pwlq_block::norm_block(*a, (hipStream_t)stream);
    return launch_status("norm launch");
}

size_t pwlq_norm_block_backward_workspace_bytes(int64_t T, int64_t D, int64_t gate_rows)
{
    if (T < 0 || T > kMostRows || D < 1 || D > 16384 || gate_rows < 0 || gate_rows > T) return 0;
    return pwlq_block::norm_backward_workspace(T, D, gate_rows);
}

int pwlq_norm_block_backward(const pwlq_norm_backward_args *a, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_sizes(a->T, a->D, 16384)) return rc;
    if (int rc = check_gate(a->gate, a->gate_rows, a->T)) return rc;
    if (!a->pre_weight || !a->d_pre) return fail(PWLQ_ENULL, "pre_weight or d_pre is NULL");
    if (!a->post_weight != !a->d_post || !a->gate != !a->d_gate)
        return fail(PWLQ_ENULL, "a weight or gate without its gradient, or a gradient without it");
    if (a->T) {
        if (int rc = check_rows("x_out", a->x_out, a->D, true)) return rc;
        if (int rc = check_rows("dx", a->dx, a->D, false)) return rc;
        const bool kept = a->x_out.type == PWLQ_I8;
        int type = a->dx.type;
        if (a->f.data) {
            if (int rc = check_rows("f", a->f, a->D, true)) return rc;
            if (int rc = check_rows("df", a->df, a->D, false)) return rc;
            type = a->df.type;
            if ((a->f.type == PWLQ_I8) != kept) return fail(PWLQ_EINVAL, "x_out and f are both of 8 bits, or neither");
            if (!kept && a->f.type != type) return fail(PWLQ_EINVAL, "f and df have one type");
        } else if (a->post_weight || a->gate) {
            return fail(PWLQ_EINVAL, "post_weight and gate go with f");
        }
        if (!kept && a->x_out.type != a->dx.type) return fail(PWLQ_EINVAL, "x_out and dx have one type");
        if (a->dx_out.data) {
            if (int rc = check_rows("dx_out", a->dx_out, a->D, false)) return rc;
            if (a->dx_out.type != a->dx.type) return fail(PWLQ_EINVAL, "dx_out and dx have one type");
        }
        if (a->du.data) {
            if (int rc = check_rows("du", a->du, a->D, false)) return rc;
            if (a->f.data && a->du.type != type) return fail(PWLQ_EINVAL, "du and df have one type");
            type = a->du.type;
        }
        if (a->dx.type != type && a->dx.type != PWLQ_F32) return fail(PWLQ_EINVAL, "dx has du's type or PWLQ_F32");
        if (int rc = check_room(workspace, workspace_bytes, pwlq_block::norm_backward_workspace(a->T, a->D, a->gate ? a->gate_rows : 0))) return rc;
    }
    pwlq_block::norm_backward(*a, workspace, (hipStream_t)stream);
    return launch_status("norm backward launch");
}

size_t pwlq_adapter_workspace_bytes(int64_t T, int64_t K, int R)
{
    if (T < 0 || T > kMostRows || K < 1 || K > 1 << 20 || R < 1 || R > 256) return 0;
    return pwlq_block::adapter_workspace(T, K, R);
}

int pwlq_adapter(const pwlq_adapter_args *a, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_adapter(a->T, a->K, a->N, a->R, a->adapters, a->weight_type, a->down, a->up, a->ids, a->scale)) return rc;
    if (a->T == 0) return PWLQ_OK;
    if (int rc = check_columns("x", a->x, a->K, a->weight_type, true)) return rc;
    if (a->base.data)
        if (int rc = check_columns("base", a->base, a->N, a->weight_type, false, true)) return rc;
    if (int rc = check_columns("out", a->out, a->N, a->weight_type)) return rc;
    if (!a->h) return fail(PWLQ_ENULL, "h is NULL");
    if (int rc = check_room(workspace, workspace_bytes, pwlq_block::adapter_workspace(a->T, a->K, a->R))) return rc;
    pwlq_block::adapter_forward(*a, workspace, (hipStream_t)stream);
    return launch_status("adapter launch");
}

size_t pwlq_adapter_backward_workspace_bytes(int64_t T, int64_t K, int64_t N, int R, int adapters)
{
    if (T < 0 || T > kMostRows || K < 1 || K > 1 << 20 || N < 1 || N > 1 << 20 || R < 1 || R > 256 || adapters < 1 || adapters > 65535)
        return 0;
    return pwlq_block::adapter_backward_workspace(T, K, N, R, adapters);
}

int pwlq_adapter_backward(const pwlq_adapter_backward_args *a, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_adapter(a->T, a->K, a->N, a->R, a->adapters, a->weight_type, a->down, a->up, a->ids, a->scale)) return rc;
    if (!a->d_down || !a->d_up) return fail(PWLQ_ENULL, "an output pointer is NULL");
    if (a->T) {
        if (int rc = check_rows("dy", a->dy, a->N, false)) return rc;
        if (a->dy.type != a->weight_type) return fail(PWLQ_EINVAL, "dy has the weights' type");
        if (int rc = check_columns("x", a->x, a->K, a->weight_type, true)) return rc;
        if (a->dx_base.data)
            if (int rc = check_columns("dx_base", a->dx_base, a->K, a->weight_type)) return rc;
        if (int rc = check_columns("dx", a->dx, a->K, a->weight_type)) return rc;
        if (!a->h) return fail(PWLQ_ENULL, "h is NULL");
        if (int rc = check_room(workspace, workspace_bytes, pwlq_block::adapter_backward_workspace(a->T, a->K, a->N, a->R, a->adapters)))
            return rc;
    }
    pwlq_block::adapter_backward(*a, workspace, (hipStream_t)stream);
    return launch_status("adapter backward launch");
}

} // extern "C"
