// The entry points of pwlq_attention.h: checks of their arguments, then the launches of launch.h.
#pragma once

#include "launch.h"

namespace {

constexpr int64_t kMostCalled = 1LL << 20;     // rows, sequences
constexpr int kMostHeads = 1024;
constexpr int64_t kMostSlots = 1LL << 30;      // of a sequence: sums of slots, tiles and windows stay within 32 bits

int check_cache(const pwlq_cache &c)
{
    if (c.type != PWLQ_BF16 && c.type != PWLQ_F16 && c.type != PWLQ_I8) return fail(PWLQ_EINVAL, "a cache has type %d, not taken here", c.type);
    if (c.D < 16 || c.D > 256 || c.D % 16 != 0) return fail(PWLQ_EINVAL, "D=%d: multiples of 16 up to 256 are taken", c.D);
    if (c.page < 16 || c.page > 65536 || (c.page & (c.page - 1)) != 0) return fail(PWLQ_EINVAL, "page=%d: powers of two from 16 to 65536 are taken", c.page);
    if (c.heads < 1 || c.heads > kMostHeads) return fail(PWLQ_EINVAL, "heads=%d outside [1,%d]", c.heads, kMostHeads);
    if (c.pages < 0 || c.pages > INT32_MAX) return fail(PWLQ_EINVAL, "pages=%lld outside [0,2^31)", (long long)c.pages);
    return PWLQ_OK;
}
int check_batch(const pwlq_batch &b, const pwlq_cache &c)
{
    if (b.T < 0 || b.T > kMostCalled) return fail(PWLQ_EINVAL, "T=%lld outside [0,%lld]", (long long)b.T, (long long)kMostCalled);
    if (b.S < 0 || b.S > kMostCalled) return fail(PWLQ_EINVAL, "S=%lld outside [0,%lld]", (long long)b.S, (long long)kMostCalled);
    if (!b.starts && b.T != b.S) return fail(PWLQ_EINVAL, "without starts T=%lld is not S=%lld", (long long)b.T, (long long)b.S);
    if (b.table_pages < 0 || b.table_pages > kMostSlots / c.page) return fail(PWLQ_EINVAL, "table_pages=%lld: a sequence of more than 2^30 rows", (long long)b.table_pages);
    return PWLQ_OK;
}
// What is read of both once there are rows.
int check_memory(const pwlq_cache &c, const pwlq_batch &b)
{
    if (!c.keys || !c.values || !b.table || !b.lengths) return fail(PWLQ_ENULL, "keys, values, table or lengths is NULL");
    if (c.type == PWLQ_I8 && (!c.key_step || !c.value_step)) return fail(PWLQ_ENULL, "the cache is of 8 bits and has no steps");
    if (c.type != PWLQ_I8 && (c.key_step || c.value_step)) return fail(PWLQ_EINVAL, "the cache is not of 8 bits and has steps");
    if (((uintptr_t)c.keys | (uintptr_t)c.values | (uintptr_t)c.key_step | (uintptr_t)c.value_step) % 16 != 0)
        return fail(PWLQ_EINVAL, "the cache is not aligned to 16 bytes");
    if (((uintptr_t)b.table | (uintptr_t)b.lengths | (uintptr_t)b.starts) % 4 != 0) return fail(PWLQ_EINVAL, "table, lengths or starts is not aligned");
    if (c.pages < 1 || b.table_pages < 1) return fail(PWLQ_EINVAL, "a cache or a table without pages");
    if (b.table_stride < b.table_pages && b.S > 1) return fail(PWLQ_EINVAL, "table_stride=%lld for %lld pages", (long long)b.table_stride, (long long)b.table_pages);
    return PWLQ_OK;
}
int check_heads(const char *name, const pwlq_heads &h, int heads, const pwlq_cache &c, int64_t T, int type, bool output)
{
    if (!h.data) return fail(PWLQ_ENULL, "%s is NULL", name);
    if (h.type != PWLQ_BF16 && h.type != PWLQ_F16) return fail(PWLQ_EINVAL, "%s has type %d, not taken here", name, h.type);
    if (h.type != type || (c.type != PWLQ_I8 && c.type != type)) return fail(PWLQ_EINVAL, "%s has type %d beside others", name, h.type);
    if ((uintptr_t)h.data % 2 != 0) return fail(PWLQ_EINVAL, "%s is not aligned to its elements", name);
    constexpr int64_t most = 1LL << 40;
    if (h.stride < 0 || h.head_stride < 0 || h.stride > most || h.head_stride > most) return fail(PWLQ_EINVAL, "%s has a stride that is not taken", name);
    const bool apart = (heads == 1 || h.head_stride >= c.D) && (T == 1 || h.stride >= c.D) &&
                       (heads == 1 || T == 1 || h.stride >= (heads - 1) * h.head_stride + c.D || h.head_stride >= (T - 1) * h.stride + c.D);
    if (output && !apart) return fail(PWLQ_EINVAL, "%s: rows overlap", name);
    return PWLQ_OK;
}
int check_query_heads(int q_heads, int heads)
{
    if (q_heads < heads || q_heads > kMostHeads || q_heads % heads != 0)
        return fail(PWLQ_EINVAL, "q_heads=%d: a multiple of the cache's %d up to %d is taken", q_heads, heads, kMostHeads);
    return PWLQ_OK;
}
int check_attend(const pwlq_attend_args *a)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_cache(a->cache)) return rc;
    if (int rc = check_batch(a->batch, a->cache)) return rc;
    if (int rc = check_query_heads(a->q_heads, a->cache.heads)) return rc;
    if (a->longest < 0) return fail(PWLQ_EINVAL, "longest=%lld is negative", (long long)a->longest);
    return PWLQ_OK;
}

} // namespace

extern "C" {

int pwlq_append(const pwlq_append_args *a, void *stream)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_cache(a->cache)) return rc;
    if (int rc = check_batch(a->batch, a->cache)) return rc;
    if (a->rotated < 0 || a->rotated > a->cache.D || a->rotated % 16 != 0)
        return fail(PWLQ_EINVAL, "rotated=%d: multiples of 16 up to D=%d are taken", a->rotated, a->cache.D);
    if (a->q.data) {
        if (int rc = check_query_heads(a->q_heads, a->cache.heads)) return rc;
    } else if (a->q_heads || a->q_out.data) {
        return fail(PWLQ_ENULL, "q_heads and q_out go with q");
    }
    if (a->batch.T == 0 || a->batch.S == 0) return PWLQ_OK;
    if (int rc = check_memory(a->cache, a->batch)) return rc;
    const int type = a->k.type;
    if (int rc = check_heads("k", a->k, a->cache.heads, a->cache, a->batch.T, type, false)) return rc;
    if (int rc = check_heads("v", a->v, a->cache.heads, a->cache, a->batch.T, type, false)) return rc;
    if (a->q.data) {
        if (int rc = check_heads("q", a->q, a->q_heads, a->cache, a->batch.T, type, false)) return rc;
        if (int rc = check_heads("q_out", a->q_out, a->q_heads, a->cache, a->batch.T, type, true)) return rc;
    }
    if (a->rotated && !a->frequencies) return fail(PWLQ_ENULL, "frequencies is NULL");
    if (((uintptr_t)a->frequencies | (uintptr_t)a->positions) % 4 != 0) return fail(PWLQ_EINVAL, "frequencies or positions is not aligned");
    pwlq_attention::append(*a, (hipStream_t)stream);
    return launch_status("append launch");
}

int pwlq_read(const pwlq_read_args *a, void *stream)
{
    if (!a) return fail(PWLQ_ENULL, "args is NULL");
    if (int rc = check_cache(a->cache)) return rc;
    if (int rc = check_batch(a->batch, a->cache)) return rc;
    if (a->batch.T == 0 || a->batch.S == 0) return PWLQ_OK;
    if (int rc = check_memory(a->cache, a->batch)) return rc;
    if (!a->k.data && !a->v.data) return fail(PWLQ_ENULL, "k and v are both NULL");
    const int type = a->k.data ? a->k.type : a->v.type;
    if (a->k.data)
        if (int rc = check_heads("k", a->k, a->cache.heads, a->cache, a->batch.T, type, true)) return rc;
    if (a->v.data)
        if (int rc = check_heads("v", a->v, a->cache.heads, a->cache, a->batch.T, type, true)) return rc;
    pwlq_attention::read(*a, (hipStream_t)stream);
    return launch_status("read launch");
}

size_t pwlq_attend_workspace_bytes(const pwlq_attend_args *a)
{
    if (check_attend(a) || a->batch.T == 0 || a->batch.S == 0) return 0;
    return pwlq_attention::attend_workspace(*a);
}

int pwlq_attend(const pwlq_attend_args *a, void *workspace, size_t workspace_bytes, void *stream)
{
    if (int rc = check_attend(a)) return rc;
    // beyond these the factors that the kernels make of them are no numbers of binary32
    constexpr float most = (float)(1LL << 60);
    if (!(a->scale >= -most && a->scale <= most)) return fail(PWLQ_EINVAL, "scale=%g outside [-2^60,2^60]", (double)a->scale);
    if (a->cap != 0.0f && !(a->cap >= 1.0f / most && a->cap <= most)) return fail(PWLQ_EINVAL, "cap=%g is neither 0 nor within [2^-60,2^60]", (double)a->cap);
    if (a->window < 0) return fail(PWLQ_EINVAL, "window=%lld is negative", (long long)a->window);
    if (a->tree && (a->slopes || a->window || a->prefix)) return fail(PWLQ_EINVAL, "a tree goes without slopes, window and prefix");
    if (a->tree && (a->tree_words < 1 || a->tree_words > kMostCalled / 64))
        return fail(PWLQ_EINVAL, "tree_words=%lld outside [1,%lld]", (long long)a->tree_words, (long long)(kMostCalled / 64));
    if (a->batch.T == 0 || a->batch.S == 0) return PWLQ_OK;
    if (int rc = check_memory(a->cache, a->batch)) return rc;
    if (int rc = check_heads("q", a->q, a->q_heads, a->cache, a->batch.T, a->q.type, false)) return rc;
    if (int rc = check_heads("out", a->out, a->q_heads, a->cache, a->batch.T, a->q.type, true)) return rc;
    if (((uintptr_t)a->slopes | (uintptr_t)a->prefix) % 4 != 0 || (uintptr_t)a->tree % 8 != 0)
        return fail(PWLQ_EINVAL, "slopes, prefix or tree is not aligned");
    if (int rc = check_room(workspace, workspace_bytes, pwlq_attention::attend_workspace(*a))) return rc;
    pwlq_attention::attend(*a, workspace, (hipStream_t)stream);
    return launch_status("attention launch");
}

} // extern "C"
