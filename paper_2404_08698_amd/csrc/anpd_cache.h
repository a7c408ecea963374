// A sequence's paged cache as the library's translation units share it (host side).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <vector>

#include "anpd_common.h"

#define HIP_TRY(expr)                                                                             \
    do {                                                                                          \
        hipError_t e_ = (expr);                                                                   \
        if (e_ != hipSuccess) return fail(ANPD_E_HIP, "%s: %s", #expr, hipGetErrorString(e_));    \
    } while (0)

namespace anpd {

inline size_t align_up(size_t x, size_t a = 256) { return (x + a - 1) / a * a; }

// What a page holds, and how.
struct CacheShape {
    int32_t n_layers, n_heads, n_kv_heads, head_dim, dtype, page_tokens;
    bool fragments;   // matrix-core order inside a block (bf16, 16 tokens a page); otherwise [token][dim]

    size_t page_bytes() const
    {
        return (size_t)n_layers * 2 * n_kv_heads * head_dim * page_tokens * (dtype == ANPD_BF16 ? 2 : 4);
    }
    size_t pool_bytes(int32_t max_tokens) const
    {
        const size_t pages = (size_t)(max_tokens + page_tokens - 1) / page_tokens;
        return align_up(pages * page_bytes()) + align_up((pages + 1) * sizeof(int32_t));
    }
};

}  // namespace anpd

struct anpd_kv {
    const anpd_model *m;             // NULL: a cache without a model
    anpd::CacheShape shape;
    int device, n_cu;                // where the pool lies, and its compute units
    char *pool;
    int32_t n_pages, max_tokens, len;
    std::vector<int32_t> table;      // logical -> physical, -1 = none
    std::vector<int32_t> dev_table;  // what the device copy currently holds
    std::vector<int32_t> free_list;  // physical pages, handed out from the back
    int32_t *d_table, *d_len;
    int32_t *pin;                    // pinned staging: [0] length, [1..] table
    bool table_dirty;
    // prompts whose last rows' weights are wanted (anpd_kv_observe)
    float *seen_mass;
    int64_t seen_ld;
    int32_t seen_rows;
    char *seen_ws;
};

namespace anpd {

// Make sure logical pages covering positions [0, upto) exist; refresh the device table if needed.
int32_t ensure_pages(anpd_kv *kv, int32_t upto, hipStream_t st);
// Return pages wholly beyond `len` to the free list.
void release_pages(anpd_kv *kv, int32_t len);
// A cache in caller-owned device memory (checked by the caller of this); `who` names the entry point in messages.
int32_t make_cache(const char *who, const anpd_model *m, const CacheShape &shape, void *pool, size_t pool_bytes, int32_t max_tokens, anpd_kv **out);

// Adds the weights of the last rows of a prompt of P rows, whose queries are the split operand qp of G row groups, to the cache's
// observed mass of this layer (their keys are cached, the length is still that before the prompt).
int32_t observe_layer(const anpd_kv *kv, int32_t layer, const void *qp, int32_t G, int32_t P, hipStream_t st);

}  // namespace anpd
