// Rows of keys and values into caches and back, the commit of a tree's path, and attention over caches of 8 bits: host half.  The kernels and their
// reasons are in anpd_cache_rows.h and anpd_cache_attn8.h.
#include <hip/hip_runtime.h>

#include <cstring>

#include "anpd_cache.h"
#include "anpd_cache_attn8.h"
#include "anpd_cache_rows.h"

using namespace anpd;

namespace {

CacheKind kind_of(const CacheShape &c)
{
    return c.dtype == ANPD_INT8 ? kCache8 : c.fragments ? kCacheFragments : c.dtype == ANPD_BF16 ? kCacheBf16 : kCacheF32;
}

// The sequences, rows and arrays of a call, checked, as the kernels take them.
int32_t gather(const char *who, const anpd_kv *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, const void *k, int64_t ldk,
               const void *v, int64_t ldv, int32_t dtype, bool store, RowsArgs &a)
{
    if (!kvs || !n_rows) return fail(ANPD_E_INVAL, "%s: NULL argument", who);
    if (n_seq < 1 || n_seq > kAttnMaxSeqs) return fail(ANPD_E_INVAL, "%s: n_seq must be in 1..%d", who, kAttnMaxSeqs);
    for (int s = 0; s < n_seq; ++s)
        if (!kvs[s]) return fail(ANPD_E_INVAL, "%s: NULL cache", who);
    const CacheShape &c = kvs[0]->shape;
    if (c.head_dim != 64 && c.head_dim != 128) return fail(ANPD_E_INVAL, "%s: head_dim must be 64 or 128", who);
    if (layer < 0 || layer >= c.n_layers) return fail(ANPD_E_INVAL, "%s: layer %d outside [0, %d)", who, layer, c.n_layers);
    if (dtype != ANPD_F32 && dtype != ANPD_BF16) return fail(ANPD_E_INVAL, "%s: unknown dtype", who);
    const int64_t width = (int64_t)c.n_kv_heads * c.head_dim;
    if (ldk < width || ldv < width) return fail(ANPD_E_INVAL, "%s: rows are %lld elements wide and %lld and %lld apart", who, (long long)width, (long long)ldk, (long long)ldv);
    std::memset(&a, 0, sizeof(a));
    int64_t rows = 0, spans = 0;
    for (int s = 0; s < n_seq; ++s) {
        const anpd_kv *kv = kvs[s];
        if (!(kv->shape == c) || kv->device != kvs[0]->device) return fail(ANPD_E_INVAL, "%s: cache %d has another shape or device than the first", who, s);
        for (int t = 0; store && t < s; ++t)
            if (kvs[t] == kv) return fail(ANPD_E_INVAL, "%s: sequences %d and %d share a cache", who, t, s);
        const int32_t n = n_rows[s], at = pos0 ? pos0[s] : kv->len;
        if (n < 0 || at < 0) return fail(ANPD_E_INVAL, "%s: sequence %d: %d rows from position %d on", who, s, n, at);
        if ((int64_t)at + n > kv->max_tokens)
            return fail(ANPD_E_CAPACITY, "%s: sequence %d: position %d + %d rows exceeds capacity %d", who, s, at, n, kv->max_tokens);
        if (!store && n > 0 && kv->table[(size_t)((at + n - 1) / c.page_tokens)] < 0)
            return fail(ANPD_E_INVAL, "%s: sequence %d: position %d has no page", who, s, at + n - 1);
        a.seq[s] = {kv->pool, kv->d_table, at, n, (int32_t)rows, (int32_t)spans};
        rows += n;
        if (n > 0) spans += (at + n - 1) / 16 - at / 16 + 1;
    }
    // (fewer than 2^32 threads: two waves for each span and head)
    if (rows >= (1 << 30) || spans * c.n_kv_heads > (1ll << 25) - 2) return fail(ANPD_E_CAPACITY, "%s: too many rows", who);
    a.n_seq = n_seq;
    a.n_spans = (int32_t)spans;
    if (rows == 0) return ANPD_OK;
    if (!k || !v) return fail(ANPD_E_INVAL, "%s: NULL rows", who);
    const uintptr_t bits = (uintptr_t)k | (uintptr_t)v;
    if ((bits & (dtype == ANPD_F32 ? 3 : 1)) != 0) return fail(ANPD_E_INVAL, "%s: rows are not aligned to their type", who);
    a.k = const_cast<void *>(k);   // (store: read only)
    a.v = const_cast<void *>(v);
    a.ldk = ldk;
    a.ldv = ldv;
    a.layer = layer;
    a.n_layers = c.n_layers;
    a.n_kv_heads = c.n_kv_heads;
    a.page_tokens = c.page_tokens;
    a.wide = (bits & 15) == 0 && (ldk | ldv) % (dtype == ANPD_F32 ? 4 : 8) == 0;
    return ANPD_OK;
}

template <int KIND, bool STORE, typename T>
void launch_kind(const RowsArgs &a, int head_dim, dim3 grid, hipStream_t st)
{
    if (head_dim == 128) hipLaunchKernelGGL((cache_rows_kernel<KIND, 128, STORE, T>), grid, dim3(64 * kRowsWaves), 0, st, a);
    else hipLaunchKernelGGL((cache_rows_kernel<KIND, 64, STORE, T>), grid, dim3(64 * kRowsWaves), 0, st, a);
}
template <bool STORE, typename T>
int32_t launch_rows(const RowsArgs &a, const CacheShape &c, hipStream_t st)
{
    const dim3 grid((unsigned)(((int64_t)a.n_spans * a.n_kv_heads * 2 + kRowsWaves - 1) / kRowsWaves));
    switch (kind_of(c)) {
    case kCache8: launch_kind<kCache8, STORE, T>(a, c.head_dim, grid, st); break;
    case kCacheFragments: launch_kind<kCacheFragments, STORE, T>(a, c.head_dim, grid, st); break;
    case kCacheBf16: launch_kind<kCacheBf16, STORE, T>(a, c.head_dim, grid, st); break;
    default: launch_kind<kCacheF32, STORE, T>(a, c.head_dim, grid, st);
    }
    HIP_TRY(hipGetLastError());
    return ANPD_OK;
}
template <bool STORE>
int32_t launch_rows(const RowsArgs &a, const CacheShape &c, int32_t dtype, hipStream_t st)
{
    return dtype == ANPD_F32 ? launch_rows<STORE, float>(a, c, st) : launch_rows<STORE, bf16_t>(a, c, st);
}

template <int KIND>
void launch_commit(const CommitArgs &a, int head_dim, dim3 grid, hipStream_t st)
{
    if (head_dim == 128) hipLaunchKernelGGL((cache_commit_kernel<KIND, 128>), grid, dim3(128), 0, st, a);
    else hipLaunchKernelGGL((cache_commit_kernel<KIND, 64>), grid, dim3(64), 0, st, a);
}

template <int DH, int TERMS>
void launch8(const AttnArgs &a, Seen rules, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.n_blocks * a.n_splits * a.n_kv_heads));
    if (rules == kTree) hipLaunchKernelGGL((cache_attn8_kernel<DH, TERMS, kTree>), grid, dim3(256), 0, st, a);
    else if (rules == kRuled) hipLaunchKernelGGL((cache_attn8_kernel<DH, TERMS, kRuled>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((cache_attn8_kernel<DH, TERMS, kCausal>), grid, dim3(256), 0, st, a);
}

}  // namespace

namespace anpd {

void launch_attention8(const AttnArgs &a, Seen rules, int head_dim, hipStream_t st)
{
    if (head_dim == 128) { if (a.q_f32) launch8<128, 2>(a, rules, st); else launch8<128, 1>(a, rules, st); }
    else if (a.q_f32) launch8<64, 2>(a, rules, st);
    else launch8<64, 1>(a, rules, st);
}

int32_t copy_rows8(const anpd_kv *kv, int32_t layer, int32_t pos0, int32_t n, float *k, float *v, bool to_cache, hipStream_t st)
{
    RowsArgs a;
    const int64_t width = (int64_t)kv->shape.n_kv_heads * kv->shape.head_dim;
    const int32_t rc = gather("anpd_kv_read/write", &kv, 1, &n, &pos0, layer, k, width, v, width, ANPD_F32, to_cache, a);
    if (rc != ANPD_OK) return rc;
    return to_cache ? launch_rows<true>(a, kv->shape, ANPD_F32, st) : launch_rows<false>(a, kv->shape, ANPD_F32, st);
}

}  // namespace anpd

extern "C" {

int32_t anpd_kv_store(anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, const void *k, int64_t ldk, const void *v,
                      int64_t ldv, int32_t dtype, void *stream)
{
    const char *who = "anpd_kv_store";
    RowsArgs a;
    int32_t rc = gather(who, kvs, n_seq, n_rows, pos0, layer, k, ldk, v, ldv, dtype, true, a);
    if (rc != ANPD_OK || a.n_spans == 0) return rc;
    const CacheShape &c = kvs[0]->shape;
    OnDevice on;
    if ((rc = on.enter(who, kvs[0]->device)) != ANPD_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    // Pages that are not there yet: their table goes through the cache's pinned memory, which the next call may use.
    bool wait = false;
    for (int s = 0; s < n_seq; ++s) {
        const SeqView &v = a.seq[s];
        if (v.n == 0) continue;
        anpd_kv *kv = kvs[s];
        if (kv->table_dirty || kv->table[(size_t)((v.pos0 + v.n - 1) / c.page_tokens)] < 0) {
            if (!wait) {
                hipStreamCaptureStatus status;
                HIP_TRY(hipStreamIsCapturing(st, &status));
                if (status != hipStreamCaptureStatusNone) return fail(ANPD_E_INVAL, "%s: sequence %d has no page for its rows, and the stream is captured", who, s);
                wait = true;
            }
            if ((rc = ensure_pages(kv, v.pos0 + v.n, st)) != ANPD_OK) break;
        }
    }
    if (rc == ANPD_OK) rc = launch_rows<true>(a, c, dtype, st);
    if (wait) HIP_TRY(hipStreamSynchronize(st));
    return rc;
}

int32_t anpd_kv_load(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, void *k, int64_t ldk, void *v,
                     int64_t ldv, int32_t dtype, void *stream)
{
    const char *who = "anpd_kv_load";
    RowsArgs a;
    int32_t rc = gather(who, kvs, n_seq, n_rows, pos0, layer, k, ldk, v, ldv, dtype, false, a);
    if (rc != ANPD_OK || a.n_spans == 0) return rc;
    OnDevice on;
    if ((rc = on.enter(who, kvs[0]->device)) != ANPD_OK) return rc;
    return launch_rows<false>(a, kvs[0]->shape, dtype, (hipStream_t)stream);
}

int32_t anpd_kv_commit(anpd_kv_t *kv, const int32_t *rows, int32_t n, void *stream)
{
    const char *who = "anpd_kv_commit";
    if (!kv || (!rows && n != 0)) return fail(ANPD_E_INVAL, "%s: NULL argument", who);
    const CacheShape &c = kv->shape;
    if (c.head_dim != 64 && c.head_dim != 128) return fail(ANPD_E_INVAL, "%s: head_dim must be 64 or 128", who);
    if (n < 0 || n > kTreeRows) return fail(ANPD_E_INVAL, "%s: %d rows, 0..%d are possible", who, n, kTreeRows);
    CommitArgs a;
    std::memset(&a, 0, sizeof(a));
    bool moves = false;
    for (int i = 0; i < n; ++i) {
        if (rows[i] < 0 || rows[i] >= kTreeRows || (i > 0 && rows[i] <= rows[i - 1])) return fail(ANPD_E_INVAL, "%s: rows must ascend in 0..%d", who, kTreeRows - 1);
        a.slot[i] = (uint8_t)rows[i];
        moves = moves || rows[i] != i;
    }
    if (n > 0) {
        if ((int64_t)kv->len + rows[n - 1] >= kv->max_tokens) return fail(ANPD_E_CAPACITY, "%s: position %d + row %d exceeds capacity %d", who, kv->len, rows[n - 1], kv->max_tokens);
        if (kv->table[(size_t)((kv->len + rows[n - 1]) / c.page_tokens)] < 0) return fail(ANPD_E_INVAL, "%s: position %d has no page", who, kv->len + rows[n - 1]);
    }
    OnDevice on;
    int32_t rc = on.enter(who, kv->device);
    if (rc != ANPD_OK) return rc;
    if (moves) {
        a.pool = kv->pool;
        a.table = kv->d_table;
        a.len = kv->len;
        a.n = n;
        a.n_layers = c.n_layers;
        a.n_kv_heads = c.n_kv_heads;
        a.page_tokens = c.page_tokens;
        const dim3 grid((unsigned)(c.n_layers * c.n_kv_heads), 2);
        hipStream_t st = (hipStream_t)stream;
        switch (kind_of(c)) {
        case kCache8: launch_commit<kCache8>(a, c.head_dim, grid, st); break;
        case kCacheFragments: launch_commit<kCacheFragments>(a, c.head_dim, grid, st); break;
        case kCacheBf16: launch_commit<kCacheBf16>(a, c.head_dim, grid, st); break;
        default: launch_commit<kCacheF32>(a, c.head_dim, grid, st);
        }
        HIP_TRY(hipGetLastError());
    }
    return anpd_kv_truncate(kv, kv->len + n, stream);
}

}  // extern "C"
