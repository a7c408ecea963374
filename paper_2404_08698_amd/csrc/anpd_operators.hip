// Operators on caches: host half (arguments, how the work is divided, launches).  The kernels and their reasons are in
// anpd_cache_attn.h and anpd_cache_evict.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "anpd_cache.h"
#include "anpd_cache_attn.h"
#include "anpd_cache_attn8.h"
#include "anpd_cache_evict.h"

using namespace anpd;

namespace {

// What anpd_attention and anpd_key_mass have in common: the sequences and rules, checked, as the kernels take them.
int32_t gather(const char *who, const anpd_kv *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, const int32_t *parent,
               const anpd_attn_rules *rules, AttnArgs &a, int64_t &rows)
{
    if (!kvs || !n_rows) return fail(ANPD_E_INVAL, "%s: NULL argument", who);
    if (n_seq < 1 || n_seq > kAttnMaxSeqs) return fail(ANPD_E_INVAL, "%s: n_seq must be in 1..%d", who, kAttnMaxSeqs);
    for (int s = 0; s < n_seq; ++s)
        if (!kvs[s]) return fail(ANPD_E_INVAL, "%s: NULL cache", who);
    const CacheShape &c = kvs[0]->shape;
    std::memset(&a, 0, sizeof(a));
    a.n_seq = n_seq;
    a.n_layers = c.n_layers;
    a.n_heads = c.n_heads;
    a.n_kv_heads = c.n_kv_heads;
    a.group = c.n_heads / c.n_kv_heads;
    a.page_tokens = c.page_tokens;
    a.scale = 1.0f / std::sqrt((float)c.head_dim);
    a.parent = parent;
    rows = 0;
    for (int s = 0; s < n_seq; ++s) {
        const anpd_kv *kv = kvs[s];
        if (!(kv->shape == c) || kv->device != kvs[0]->device) return fail(ANPD_E_INVAL, "%s: cache %d has another shape or device than the first", who, s);
        const int32_t n = n_rows[s], at = pos0 ? pos0[s] : kv->len;
        if (n < 0 || at < 0) return fail(ANPD_E_INVAL, "%s: sequence %d: %d rows from position %d on", who, s, n, at);
        if ((int64_t)at + n > kv->max_tokens)
            return fail(ANPD_E_CAPACITY, "%s: sequence %d: position %d + %d rows exceeds capacity %d", who, s, at, n, kv->max_tokens);
        // (pages are given from the first position on and taken from the last: the last row's is there only with all before it)
        if (n > 0 && kv->table[(size_t)((at + n - 1) / c.page_tokens)] < 0)
            return fail(ANPD_E_INVAL, "%s: sequence %d: position %d has no page", who, s, at + n - 1);
        if ((int64_t)n * a.group >= (1 << 30)) return fail(ANPD_E_CAPACITY, "%s: sequence %d has too many rows", who, s);
        if (parent && n > kTreeRows) return fail(ANPD_E_CAPACITY, "%s: sequence %d: a tree of %d rows, %d at most", who, s, n, kTreeRows);
        a.seq[s] = {kv->pool, kv->d_table, at, n, (int32_t)rows, 0};
        rows += n;
    }
    if (rows >= (1 << 30)) return fail(ANPD_E_CAPACITY, "%s: too many rows", who);
    if (rules) {
        if (!(rules->scale >= 0.f) || !(rules->cap >= 0.f) || std::isinf(rules->scale) || std::isinf(rules->cap) || rules->window < 0 || rules->prefix < 0)
            return fail(ANPD_E_INVAL, "%s: scale, cap, window and prefix must be finite and >= 0", who);
        if (rules->scale > 0.f) a.scale = rules->scale;
        a.cap = rules->cap;
        if (a.cap > 0.f) a.scale_over_cap = a.scale / a.cap;
        if (a.cap > 0.f && !std::isnormal(a.scale_over_cap)) return fail(ANPD_E_INVAL, "%s: scale / cap is beyond the range of fp32", who);
        if ((((uintptr_t)rules->slopes | (uintptr_t)rules->first_key) & 3) != 0) return fail(ANPD_E_INVAL, "%s: slopes or first_key are not aligned to their type", who);
        a.window = rules->window;
        a.prefix = rules->prefix;
        a.slopes = rules->slopes;
        a.first_key = rules->first_key;
    }
    return ANPD_OK;
}

bool ruled(const AttnArgs &a) { return a.cap > 0.f || a.slopes || a.window > 0 || a.prefix > 0 || a.first_key; }

int32_t rows_in(const char *who, const CacheShape &c, int32_t layer, const void *q, int64_t ldq, int32_t dtype, AttnArgs &a)
{
    if (layer < 0 || layer >= c.n_layers) return fail(ANPD_E_INVAL, "%s: layer %d outside [0, %d)", who, layer, c.n_layers);
    if (dtype != ANPD_F32 && dtype != ANPD_BF16) return fail(ANPD_E_INVAL, "%s: unknown dtype", who);
    const int64_t width = (int64_t)c.n_heads * c.head_dim;
    if (ldq < width) return fail(ANPD_E_INVAL, "%s: rows are %lld elements wide and %lld apart", who, (long long)width, (long long)ldq);
    if (((uintptr_t)q & (dtype == ANPD_F32 ? 3 : 1)) != 0) return fail(ANPD_E_INVAL, "%s: rows are not aligned to their type", who);
    a.layer = layer;
    a.q = q;
    a.ldq = ldq;
    a.q_f32 = dtype == ANPD_F32;
    a.q_wide = ((uintptr_t)q & 15) == 0 && ldq % (a.q_f32 ? 4 : 8) == 0;
    return ANPD_OK;
}

// ---- attention: how the work is divided

struct Plan {
    bool shared;   // many rows share keys through LDS; otherwise blocks of 32 rows
    int row_block, key_tile;
    size_t part_bytes;
};

// The key tiles of all row blocks of a sequence, and the most that a block can have.  All: by the blocks at its ends (in between it goes in a
// straight line), with a window by up to eight blocks.
void count_tiles(const AttnArgs &a, const SeqView &v, int row_block, int key_tile, int64_t &blocks, int64_t &tiles, int &most)
{
    const int64_t rows = (int64_t)v.n * a.group;
    const int total = v.pos0 + v.n, span = a.parent ? v.n : row_block / a.group;
    blocks = (rows + row_block - 1) / row_block;
    const int64_t samples = blocks < 2 ? blocks : (a.window > 0 && blocks > 2 ? (blocks < 8 ? blocks : 8) : 2);
    tiles = 0;
    for (int64_t i = 0; i < samples; ++i) {
        const int64_t from = (samples > 1 ? (blocks - 1) * i / (samples - 1) : 0) * row_block, to = from + row_block < rows ? from + row_block : rows;
        tiles += key_tiles(a, v, v.pos0 + (int)(from / a.group), v.pos0 + (int)((to - 1) / a.group), key_tile).n;
    }
    tiles = blocks * tiles / samples;
    // (a window's tiles depend on where it begins inside the first one)
    const int pre = a.prefix < total ? a.prefix : total, all = (total > pre ? total : pre) - 1;
    int64_t bound = all / key_tile + 1;
    if (a.window > 0) {
        const int64_t some = (pre + key_tile - 1) / key_tile + ((int64_t)a.window + span + 1) / key_tile + 2;
        if (some < bound) bound = some;
    }
    most = (int)bound;
}

// Sets the row blocks of a's sequences, the splits and their size, for a.q_f32.
Plan plan_attention(AttnArgs &a, const CacheShape &c, int n_cu)
{
    Plan p;
    const int shared_rows = tile_rows(a.q_f32 ? 3 : 1);
    int64_t blocks[2] = {0, 0}, tiles[2] = {0, 0};   // of either form
    int most[2] = {0, 0};
    for (int s = 0; s < a.n_seq; ++s) {
        if (a.seq[s].n == 0) continue;
        for (int form = 0; form < 2; ++form) {
            int64_t b, t;
            int m;
            count_tiles(a, a.seq[s], form ? shared_rows : kRowTile, form ? kTileKeys : kStreamTile, b, t, m);
            blocks[form] += b;
            tiles[form] += t * a.n_kv_heads;
            if (m > most[form]) most[form] = m;
        }
    }
    // The shared form, a block per compute unit: as many splits as give all of them a block, none shorter than twelve tiles.
    const int64_t shared_items = blocks[1] * a.n_kv_heads;
    int64_t splits = shared_items > 0 ? n_cu / shared_items : 1;
    if (splits > most[1] / 12) splits = most[1] / 12;
    if (splits < 1) splits = 1;
    const int64_t shared_chunk = (most[1] + splits - 1) / splits;
    // Which form, by what tiles were measured to take.  Blocks of 32 rows: a tile of 128 keys 0.95 us of a compute unit (fp32 rows 1.7), and four to
    // begin with.  Shared: a tile of 32 keys 0.9 us (1.28) of the longest block, 1.1 (1.45) of a unit where there are many, 1.6 (2.5) more for those
    // that a window cuts; six to begin with, or twelve and the parts that are joined, at 4.5 TB/s.  Documents that begin behind a row's
    // first key, which are not looked at here, shorten the former more, with fp32 rows always enough.  Caps and biases are the former's: their
    // vector instructions leave nothing to share.  600 shapes (heads of 128 and 64, 1 to 16 per key head, 128 to 3584 rows, windows, prefixes, documents):
    // 2.3 % above the better one on average, heads of 128 1.2; 50 by more than a tenth, 57 % at worst (documents, heads of 64: a tile of theirs costs the
    // former less than is reckoned here).  32 heads of 128, blocks of 32 rows / shared, us: 1000 rows 24 / 35, 2000 63 / 58, 3584 160 / 112; fp32 37 / 45,
    // 109 / 99, 296 / 271; 3584 in a window of 300 68 / 75, one key head for 16 67 / 42; 3584 with a cap 252 / 315, fp32 400 / 677.
    int64_t rows = 0;
    for (int s = 0; s < a.n_seq; ++s) rows += a.seq[s].n;
    const double longest_us = (a.q_f32 ? 1.28 : 0.9) * (double)shared_chunk, all_us = (a.q_f32 ? 1.45 : 1.1) * (double)tiles[1] / n_cu;
    double shared_us = (longest_us > all_us ? longest_us : all_us) + 6.0;
    if (splits > 1) shared_us += 6.0 + (double)rows * c.n_heads * splits * c.head_dim * 4 / 4.5e6;
    if (a.window > 0) shared_us += (a.q_f32 ? 2.5 : 1.6) * (shared_rows / a.group / 32.0 + 1.0);
    if (a.first_key) shared_us *= 1.4;
    p.shared = c.fragments && !a.parent && !(a.cap > 0.f || a.slopes) && !(a.q_f32 && a.first_key) && shared_us < (a.q_f32 ? 1.7 : 0.95) * (double)tiles[0] / n_cu + 4.0;
    p.row_block = p.shared ? shared_rows : kRowTile;
    p.key_tile = p.shared ? kTileKeys : kStreamTile;
    a.n_blocks = 0;
    for (int s = 0; s < a.n_seq; ++s) {
        a.seq[s].block0 = a.n_blocks;
        a.n_blocks += (int32_t)(((int64_t)a.seq[s].n * a.group + p.row_block - 1) / p.row_block);
    }
    const int64_t items = blocks[p.shared] * a.n_kv_heads;
    const int longest = most[p.shared];
    if (p.shared) a.chunk = (int)shared_chunk;
    else {
        // Two blocks for each compute unit, of at least two tiles: a tile is about 1.3 us, joining 2.5 (32 heads of 128, 1 / 32 rows behind
        // 1000 positions 9.1 / 11.3 us, a tile each 9.7 / 14.4).  Caches in plain order, whose tiles take four times that, a tile each, and one block
        // of heads of 128, which fill a unit's registers (fp32, 4 heads of 64, 8 rows behind 1000 16 -> 13, 32 of 128, a row behind 1000 23 -> 19).
        // Caches of 8 bits the same, but up to three tiles are not split (32 heads of 128, a row / 32 rows behind 250 positions 9.6 / 10.6 -> 8.0 / 9.3); with two blocks
        // for each unit and two tiles for each: behind 1000 9.8 / 12.6 -> 10.2 / 12.8, behind 16000 30.1 / 31.0 -> 31.0 / 32.5.
        const int per_unit = c.fragments || c.head_dim == 64 ? 2 : 1, least = c.fragments || (c.dtype == ANPD_INT8 && longest <= 3) ? 2 : 1;
        splits = items > 0 ? per_unit * n_cu / items : 1;
        if (splits > longest / least) splits = longest / least;
        if (splits < 1) splits = 1;
        a.chunk = (int)((longest + splits - 1) / splits);
    }
    if (a.chunk < 1) a.chunk = 1;
    a.n_splits = longest > 0 ? (longest + a.chunk - 1) / a.chunk : 1;
    p.part_bytes = a.n_splits > 1 ? align_up((size_t)items * a.n_splits * part_floats(p.row_block, c.head_dim) * sizeof(float)) : 0;
    return p;
}

// The workspace of a call, which is the same for rows of both types.
size_t attention_part_bytes(AttnArgs a, const CacheShape &c, int n_cu)
{
    size_t need = 0;
    for (int f32 = 0; f32 < 2; ++f32) {
        a.q_f32 = f32;
        const size_t bytes = plan_attention(a, c, n_cu).part_bytes;
        if (bytes > need) need = bytes;
    }
    return need;
}

template <int DH, int TERMS, int RULES>
int32_t launch_fragments(const AttnArgs &a, const Plan &p, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.n_blocks * a.n_splits * a.n_kv_heads));
    if constexpr (RULES != kTree) if (p.shared) {
        constexpr size_t lds = tile_lds_bytes(DH);
        // (at every call: the attribute is the current device's)
        if (lds > 65536) HIP_TRY(hipFuncSetAttribute((const void *)cache_attn_tile_kernel<DH, TERMS, RULES>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        hipLaunchKernelGGL((cache_attn_tile_kernel<DH, TERMS, RULES>), grid, dim3(tile_waves(TERMS) * 64), lds, st, a);
        return ANPD_OK;
    }
    hipLaunchKernelGGL((cache_attn_stream_kernel<DH, TERMS, RULES>), grid, dim3(256), 0, st, a);
    return ANPD_OK;
}
template <int DH>
int32_t launch_attention(const AttnArgs &a, const Plan &p, const CacheShape &c, hipStream_t st)
{
    const Seen rules = a.parent ? kTree : ruled(a) ? kRuled : kCausal;
    if (c.fragments) {
#define ANPD_ATTEND(RULES) (a.q_f32 ? launch_fragments<DH, 3, RULES>(a, p, st) : launch_fragments<DH, 1, RULES>(a, p, st))
        const int32_t rc = rules == kTree ? ANPD_ATTEND(kTree) : rules == kRuled ? ANPD_ATTEND(kRuled) : ANPD_ATTEND(kCausal);
#undef ANPD_ATTEND
        if (rc != ANPD_OK) return rc;
    } else if (c.dtype == ANPD_INT8) launch_attention8(a, rules, c.head_dim, st);
    else {
        const dim3 grid((unsigned)((int64_t)a.n_blocks * a.n_splits * a.n_kv_heads));
#define ANPD_ATTEND(KT) \
    if (rules == kTree) hipLaunchKernelGGL((cache_attn_plain_kernel<KT, DH, kTree>), grid, dim3(256), 0, st, a); \
    else hipLaunchKernelGGL((cache_attn_plain_kernel<KT, DH, kRuled>), grid, dim3(256), 0, st, a)
        if (c.dtype == ANPD_BF16) { ANPD_ATTEND(bf16_t); } else { ANPD_ATTEND(float); }
#undef ANPD_ATTEND
    }
    HIP_TRY(hipGetLastError());
    if (a.part) {
        const int64_t rows = (int64_t)a.n_blocks * a.n_kv_heads * p.row_block;
        const dim3 block(256);
        // (a block per row while those are few enough to run side by side)
        if (a.n_splits > 4 && rows <= 4096) hipLaunchKernelGGL((cache_attn_join_kernel<DH, true>), dim3((unsigned)rows), block, 0, st, a, p.row_block, p.key_tile);
        else hipLaunchKernelGGL((cache_attn_join_kernel<DH, false>), dim3((unsigned)(rows / (1024 / DH))), block, 0, st, a, p.row_block, p.key_tile);
        HIP_TRY(hipGetLastError());
    }
    return ANPD_OK;
}

// ---- key mass: how the work is divided

// Sets the key blocks of a's sequences and the parts of their rows.  sets: 32-key sets per wave.
size_t plan_mass(AttnArgs &a, const CacheShape &c, int n_cu, int &sets)
{
    // most row tiles of a block of keys, and all of them together
    int most;
    int64_t all;
    auto count = [&](int keys) {
        a.n_blocks = most = 0;
        all = 0;
        for (int s = 0; s < a.n_seq; ++s) {
            SeqView &v = a.seq[s];
            v.block0 = a.n_blocks;
            if (v.n == 0) continue;
            const int total = v.pos0 + v.n, pre = a.prefix < total ? a.prefix : total, blocks = (total + keys - 1) / keys;
            a.n_blocks += blocks;
            for (int b = 0; b < blocks; ++b) {
                const RowTiles t = row_tiles(b * keys, keys, v.pos0, v.n, a.group, a.window, pre);
                all += t.t1 - t.t0;
                if (t.t1 - t.t0 > most) most = t.t1 - t.t0;
            }
        }
    };
    sets = 1;
    count(kMassKeys);
    // two sets where the rows are many: the operand of a tile is then shared by twice the keys
    if (c.fragments && most >= 16) {
        sets = 2;
        count(2 * kMassKeys);
    }
    // parts of at least eight tiles, six for each compute unit: later blocks have fewer rows than earlier ones
    int64_t chunk = (all * a.n_kv_heads + 6 * n_cu - 1) / (6 * n_cu);
    if (chunk < 8) chunk = 8;
    a.chunk = chunk < most ? (int)chunk : (most > 0 ? most : 1);
    a.n_splits = most > 0 ? (most + a.chunk - 1) / a.chunk : 1;
    return a.n_splits > 1 ? align_up((size_t)a.n_blocks * a.n_kv_heads * a.n_splits * kMassKeys * sets * sizeof(float)) : 0;
}

template <int DH, int SETS>
void launch_mass_fragments(const AttnArgs &a, const MassOut &to, dim3 grid, hipStream_t st)
{
    const bool rules = ruled(a);
    if (a.q_f32) {
        if (rules) hipLaunchKernelGGL((cache_mass_kernel<DH, 3, true, SETS>), grid, dim3(256), 0, st, a, to);
        else hipLaunchKernelGGL((cache_mass_kernel<DH, 3, false, SETS>), grid, dim3(256), 0, st, a, to);
    } else if (rules) hipLaunchKernelGGL((cache_mass_kernel<DH, 1, true, SETS>), grid, dim3(256), 0, st, a, to);
    else hipLaunchKernelGGL((cache_mass_kernel<DH, 1, false, SETS>), grid, dim3(256), 0, st, a, to);
}
template <int DH>
int32_t launch_mass(const AttnArgs &a, const MassOut &to, const CacheShape &c, int sets, hipStream_t st)
{
    const dim3 grid((unsigned)((int64_t)a.n_blocks * a.n_splits * a.n_kv_heads));
    if (c.fragments) { if (sets == 2) launch_mass_fragments<DH, 2>(a, to, grid, st); else launch_mass_fragments<DH, 1>(a, to, grid, st); }
    else if (c.dtype == ANPD_BF16) hipLaunchKernelGGL((cache_mass_plain_kernel<bf16_t, DH>), grid, dim3(256), 0, st, a, to);
    else hipLaunchKernelGGL((cache_mass_plain_kernel<float, DH>), grid, dim3(256), 0, st, a, to);
    HIP_TRY(hipGetLastError());
    if (a.part) {
        hipLaunchKernelGGL(cache_mass_join_kernel, dim3((unsigned)((int64_t)a.n_blocks * a.n_kv_heads)), dim3(kMassKeys * sets), 0, st, a, to);
        HIP_TRY(hipGetLastError());
    }
    return ANPD_OK;
}

int32_t workspace_of(const char *who, AttnArgs &a, size_t need, void *workspace, size_t workspace_bytes)
{
    if (need == 0) return ANPD_OK;
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return fail(ANPD_E_INVAL, "%s: workspace must be a 256-byte aligned device buffer", who);
    if (workspace_bytes < need) return fail(ANPD_E_CAPACITY, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
    a.part = (float *)workspace;
    return ANPD_OK;
}

bool overlap(const void *a, size_t na, const void *b, size_t nb)
{
    return (const char *)a < (const char *)b + nb && (const char *)b < (const char *)a + na;
}

// Do two arrays of `heads` rows, ld numbers apart in both, of na and nb numbers each (<= ld), share any?  Rows may lie between the other's.
bool rows_overlap(const float *a, int64_t na, const float *b, int64_t nb, int64_t heads, int64_t ld)
{
    // row i of a and row i + h of b meet where -nb < d + h ld < na: the lowest h that is not too low
    const int64_t d = ((intptr_t)b - (intptr_t)a) / (int64_t)sizeof(float), low = -nb - d;
    int64_t h = (low >= 0 ? low / ld : -((-low - 1) / ld + 1)) + 1;
    if (h < 1 - heads) h = 1 - heads;
    return h < heads && d + h * ld < na;
}

bool cache_cfg_ok(const char *who, const anpd_cache_cfg *c, int32_t max_tokens, CacheShape *out)
{
#define REQ(cond, msg) if (!(cond)) { fail(ANPD_E_INVAL, "%s: " msg, who); return false; }
    REQ(c, "cfg is NULL");
    REQ(c->n_layers >= 1 && c->n_heads >= 1, "non-positive dimension");
    REQ(c->n_kv_heads >= 0 && (c->n_kv_heads == 0 || c->n_heads % c->n_kv_heads == 0), "n_kv_heads must be 0 or divide n_heads");
    REQ(c->n_heads <= (1 << 16) && c->n_layers <= (1 << 16), "more than 2^16 heads or layers");
    REQ(c->head_dim == 64 || c->head_dim == 128, "head_dim must be 64 or 128");
    REQ(c->dtype == ANPD_F32 || c->dtype == ANPD_BF16 || c->dtype == ANPD_INT8, "dtype must be ANPD_F32, ANPD_BF16 or ANPD_INT8");
    REQ(c->dtype != ANPD_INT8 || c->page_tokens == 16, "page_tokens must be 16 for ANPD_INT8");
    REQ(c->page_tokens >= 8 && c->page_tokens <= 256 && (c->page_tokens & (c->page_tokens - 1)) == 0, "page_tokens must be a power of two in 8..256");
    REQ(max_tokens >= 1 && max_tokens <= (1 << 20), "max_tokens must be in 1..2^20");
#undef REQ
    *out = {c->n_layers, c->n_heads, c->n_kv_heads > 0 ? c->n_kv_heads : c->n_heads, c->head_dim, c->dtype, c->page_tokens,
            c->dtype == ANPD_BF16 && c->page_tokens == 16};
    return true;
}

// What an observed prompt needs per layer: queries, outputs, logarithms and a workspace that suffices at every length. Attention's: a block of
// rows per split and item, splits as plan_attention bounds them; the mass's: a sum per key and part of at least eight row tiles.
struct ObserveLayout {
    size_t q, out, lse, work, work_bytes, total;
};
ObserveLayout observe_layout(const CacheShape &c, int max_tokens, int rows, int n_cu)
{
    ObserveLayout L;
    const size_t width = (size_t)c.n_heads * c.head_dim, v = (size_t)rows * (c.n_heads / c.n_kv_heads), cu = (size_t)n_cu;
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes); return at; };
    L.q = take((size_t)rows * width * sizeof(float));
    L.out = take((size_t)rows * width * sizeof(float));
    L.lse = take((size_t)rows * c.n_heads * sizeof(float));
    const size_t few = (v + kRowTile - 1) / kRowTile * c.n_kv_heads, many = (v + tile_rows(1) - 1) / tile_rows(1) * c.n_kv_heads;
    const size_t keys = ((size_t)max_tokens + 2 * kMassKeys - 1) / (2 * kMassKeys) * (2 * kMassKeys), parts = ((v + 31) / 32 + 1 + 7) / 8;
    size_t floats = (few + 2 * cu) * part_floats(kRowTile, c.head_dim);
    const size_t shared = (many + cu) * part_floats(tile_rows(1), c.head_dim), mass = parts > 1 ? keys * c.n_kv_heads * parts : 0;
    if (shared > floats) floats = shared;
    if (mass > floats) floats = mass;
    L.work_bytes = align_up(floats * sizeof(float));
    L.work = take(L.work_bytes);
    L.total = o;
    return L;
}

// anpd_attention and anpd_tree_attention (parent: the new rows are trees).
size_t attention_workspace(const char *who, const anpd_kv *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, const int32_t *parent,
                           const anpd_attn_rules *rules)
{
    AttnArgs a;
    int64_t rows;
    if (gather(who, kvs, n_seq, n_rows, pos0, parent, rules, a, rows) != ANPD_OK) return 0;
    return attention_part_bytes(a, kvs[0]->shape, kvs[0]->n_cu);
}

int32_t attend(const char *who, const anpd_kv *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, const void *q, int64_t ldq,
               int32_t dtype, const int32_t *parent, const anpd_attn_rules *rules, void *out, int64_t ldo, float *lse, void *workspace, size_t workspace_bytes,
               void *stream)
{
    AttnArgs a;
    int64_t rows;
    int32_t rc = gather(who, kvs, n_seq, n_rows, pos0, parent, rules, a, rows);
    if (rc != ANPD_OK) return rc;
    const CacheShape &c = kvs[0]->shape;
    if ((rc = rows_in(who, c, layer, q, ldq, dtype, a)) != ANPD_OK) return rc;
    if (ldo < (int64_t)c.n_heads * c.head_dim) return fail(ANPD_E_INVAL, "%s: ldo %lld is less than a row", who, (long long)ldo);
    if (rows == 0) return ANPD_OK;
    if (!q || !out) return fail(ANPD_E_INVAL, "%s: NULL rows", who);
    if (((uintptr_t)lse & 3) != 0) return fail(ANPD_E_INVAL, "%s: lse is not aligned to its type", who);
    if (((uintptr_t)out & (a.q_f32 ? 3 : 1)) != 0) return fail(ANPD_E_INVAL, "%s: out is not aligned to its type", who);
    a.out = out;
    a.ldo = ldo;
    a.lse = lse;
    a.q_wide = a.q_wide && ((uintptr_t)out & 15) == 0 && ldo % (a.q_f32 ? 4 : 8) == 0;
    // (blocks of the last sequence begin first: the longest, so that what is left at the end is short.  32 tokens of 300 to 700 cached
    // positions 54.1 -> 50.6 us)
    std::stable_sort(a.seq, a.seq + a.n_seq, [](const SeqView &x, const SeqView &y) { return x.pos0 + x.n < y.pos0 + y.n; });
    const Plan p = plan_attention(a, c, kvs[0]->n_cu);
    if ((rc = workspace_of(who, a, p.part_bytes, workspace, workspace_bytes)) != ANPD_OK) return rc;
    OnDevice on;
    if ((rc = on.enter(who, kvs[0]->device)) != ANPD_OK) return rc;
    return c.head_dim == 128 ? launch_attention<128>(a, p, c, (hipStream_t)stream) : launch_attention<64>(a, p, c, (hipStream_t)stream);
}

}  // namespace

namespace anpd {

int32_t observe_layer(const anpd_kv *kv, int32_t layer, const void *qp, int32_t G, int32_t P, hipStream_t st)
{
    const CacheShape &c = kv->shape;
    const int rows = kv->seen_rows < P ? kv->seen_rows : P, pos0 = kv->len + P - rows;
    const ObserveLayout L = observe_layout(c, kv->max_tokens, kv->seen_rows, kv->n_cu);
    float *q = (float *)(kv->seen_ws + L.q), *lse = (float *)(kv->seen_ws + L.lse), *mass = kv->seen_mass + (size_t)layer * c.n_kv_heads * kv->seen_ld;
    const int64_t width = (int64_t)c.n_heads * c.head_dim;
    hipLaunchKernelGGL(prompt_rows_kernel, dim3((unsigned)rows, (unsigned)c.n_heads), dim3((unsigned)c.head_dim), 0, st, (const bf16_t *)qp, q, G,
                       (kv->len & 15) + P - rows, c.head_dim);
    HIP_TRY(hipGetLastError());
    const int32_t rc = anpd_attention(&kv, 1, &rows, &pos0, layer, q, width, ANPD_F32, nullptr, kv->seen_ws + L.out, width, lse, kv->seen_ws + L.work, L.work_bytes, st);
    if (rc != ANPD_OK) return rc;
    return anpd_key_mass(&kv, 1, &rows, &pos0, layer, q, width, ANPD_F32, nullptr, lse, &mass, kv->seen_ld, kv->seen_ws + L.work, L.work_bytes, st);
}

}  // namespace anpd

extern "C" {

size_t anpd_cache_pool_bytes(const anpd_cache_cfg *cfg, int32_t max_tokens)
{
    CacheShape shape;
    return cache_cfg_ok("anpd_cache_pool_bytes", cfg, max_tokens, &shape) ? shape.pool_bytes(max_tokens) : 0;
}

int32_t anpd_cache_create(const anpd_cache_cfg *cfg, void *pool, size_t pool_bytes, int32_t max_tokens, anpd_kv_t **out)
{
    if (!out) return fail(ANPD_E_INVAL, "anpd_cache_create: out is NULL");
    *out = nullptr;
    CacheShape shape;
    if (!cache_cfg_ok("anpd_cache_create", cfg, max_tokens, &shape)) return ANPD_E_INVAL;
    if (!pool) return fail(ANPD_E_INVAL, "anpd_cache_create: pool is NULL");
    return make_cache("anpd_cache_create", nullptr, shape, pool, pool_bytes, max_tokens, out);
}

size_t anpd_attention_workspace_bytes(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, const anpd_attn_rules *rules)
{
    return attention_workspace("anpd_attention_workspace_bytes", kvs, n_seq, n_rows, pos0, nullptr, rules);
}

int32_t anpd_attention(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, const void *q, int64_t ldq,
                       int32_t dtype, const anpd_attn_rules *rules, void *out, int64_t ldo, float *lse, void *workspace, size_t workspace_bytes, void *stream)
{
    return attend("anpd_attention", kvs, n_seq, n_rows, pos0, layer, q, ldq, dtype, nullptr, rules, out, ldo, lse, workspace, workspace_bytes, stream);
}

size_t anpd_tree_attention_workspace_bytes(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, const anpd_attn_rules *rules)
{
    static const int32_t some = -1;   // (a tree; which one is not looked at)
    return attention_workspace("anpd_tree_attention_workspace_bytes", kvs, n_seq, n_rows, pos0, &some, rules);
}

int32_t anpd_tree_attention(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, const void *q, int64_t ldq,
                            int32_t dtype, const int32_t *parent, const anpd_attn_rules *rules, void *out, int64_t ldo, float *lse, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    const char *who = "anpd_tree_attention";
    if (!parent) return fail(ANPD_E_INVAL, "%s: NULL parent", who);
    if (((uintptr_t)parent & 3) != 0) return fail(ANPD_E_INVAL, "%s: parent is not aligned to its type", who);
    return attend(who, kvs, n_seq, n_rows, pos0, layer, q, ldq, dtype, parent, rules, out, ldo, lse, workspace, workspace_bytes, stream);
}

size_t anpd_key_mass_workspace_bytes(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, const anpd_attn_rules *rules)
{
    AttnArgs a;
    int64_t rows;
    if (gather("anpd_key_mass_workspace_bytes", kvs, n_seq, n_rows, pos0, nullptr, rules, a, rows) != ANPD_OK) return 0;
    int sets;
    return plan_mass(a, kvs[0]->shape, kvs[0]->n_cu, sets);
}

int32_t anpd_key_mass(const anpd_kv_t *const *kvs, int32_t n_seq, const int32_t *n_rows, const int32_t *pos0, int32_t layer, const void *q, int64_t ldq,
                      int32_t dtype, const anpd_attn_rules *rules, const float *lse, float *const *mass, int64_t ld_mass, void *workspace,
                      size_t workspace_bytes, void *stream)
{
    const char *who = "anpd_key_mass";
    AttnArgs a;
    int64_t rows;
    int32_t rc = gather(who, kvs, n_seq, n_rows, pos0, nullptr, rules, a, rows);
    if (rc != ANPD_OK) return rc;
    const CacheShape &c = kvs[0]->shape;
    if (c.dtype == ANPD_INT8) return fail(ANPD_E_UNIMPLEMENTED, "%s: caches of 8 bits are not taken", who);
    if ((rc = rows_in(who, c, layer, q, ldq, dtype, a)) != ANPD_OK) return rc;
    if (rows == 0) return ANPD_OK;
    if (!q || !lse || !mass) return fail(ANPD_E_INVAL, "%s: NULL argument", who);
    if (((uintptr_t)lse & 3) != 0) return fail(ANPD_E_INVAL, "%s: lse is not aligned to its type", who);
    MassOut to;
    std::memset(&to, 0, sizeof(to));
    to.ld = ld_mass;
    for (int s = 0; s < n_seq; ++s) {
        if (a.seq[s].n == 0) continue;
        const int total = a.seq[s].pos0 + a.seq[s].n;
        if (!mass[s] || ((uintptr_t)mass[s] & 3) != 0) return fail(ANPD_E_INVAL, "%s: sequence %d: NULL mass, or not aligned to its type", who, s);
        if (ld_mass < total) return fail(ANPD_E_CAPACITY, "%s: sequence %d has %d keys, ld_mass is %lld", who, s, total, (long long)ld_mass);
        for (int t = 0; t < s; ++t) {
            if (a.seq[t].n == 0) continue;
            const int other = a.seq[t].pos0 + a.seq[t].n;
            if (rows_overlap(mass[s], total, mass[t], other, c.n_kv_heads, ld_mass))
                return fail(ANPD_E_INVAL, "%s: sequences %d and %d share mass", who, t, s);
        }
        to.mass[s] = mass[s];
    }
    a.lse = const_cast<float *>(lse);   // (read only)
    int sets;
    const size_t need = plan_mass(a, c, kvs[0]->n_cu, sets);
    if ((rc = workspace_of(who, a, need, workspace, workspace_bytes)) != ANPD_OK) return rc;
    OnDevice on;
    if ((rc = on.enter(who, kvs[0]->device)) != ANPD_OK) return rc;
    return c.head_dim == 128 ? launch_mass<128>(a, to, c, sets, (hipStream_t)stream) : launch_mass<64>(a, to, c, sets, (hipStream_t)stream);
}

size_t anpd_kv_observe_workspace_bytes(const anpd_kv_t *kv, int32_t rows)
{
    if (!kv || rows < 1 || rows > ANPD_MAX_WINDOW) {
        fail(ANPD_E_INVAL, "anpd_kv_observe_workspace_bytes: bad argument");
        return 0;
    }
    return observe_layout(kv->shape, kv->max_tokens, rows, kv->n_cu).total;
}

int32_t anpd_kv_observe(anpd_kv_t *kv, float *mass, int64_t ld_mass, int32_t rows, void *workspace, size_t workspace_bytes)
{
    const char *who = "anpd_kv_observe";
    if (!kv) return fail(ANPD_E_INVAL, "%s: NULL cache", who);
    if (!mass) {
        kv->seen_mass = nullptr;
        return ANPD_OK;
    }
    if (!kv->m) return fail(ANPD_E_INVAL, "%s: the cache has no model whose prompts could be observed", who);
    if (!kv->shape.fragments) return fail(ANPD_E_UNIMPLEMENTED, "%s: matrix-core models only", who);
    if (rows < 1 || rows > ANPD_MAX_WINDOW) return fail(ANPD_E_INVAL, "%s: rows must be in 1..%d", who, ANPD_MAX_WINDOW);
    if (ld_mass < 1 || ((uintptr_t)mass & 3) != 0) return fail(ANPD_E_INVAL, "%s: bad mass", who);
    if (!workspace || ((uintptr_t)workspace & 255) != 0) return fail(ANPD_E_INVAL, "%s: workspace must be a 256-byte aligned device buffer", who);
    const size_t need = observe_layout(kv->shape, kv->max_tokens, rows, kv->n_cu).total;
    if (workspace_bytes < need) return fail(ANPD_E_CAPACITY, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
    kv->seen_mass = mass;
    kv->seen_ld = ld_mass;
    kv->seen_rows = rows;
    kv->seen_ws = (char *)workspace;
    return ANPD_OK;
}

int32_t anpd_kv_evict(const anpd_kv_t *src, anpd_kv_t *dst, const float *mass, int64_t ld_mass, int32_t keep, int32_t first, int32_t last, float rope_base,
                      int32_t *out_kept, float *out_mass, int64_t ld_out, void *stream)
{
    const char *who = "anpd_kv_evict";
    if (!src || !dst) return fail(ANPD_E_INVAL, "%s: NULL cache", who);
    const CacheShape &c = src->shape;
    if (!(c == dst->shape) || src->device != dst->device) return fail(ANPD_E_INVAL, "%s: the caches have different shapes or devices", who);
    if (c.dtype == ANPD_INT8) return fail(ANPD_E_UNIMPLEMENTED, "%s: caches of 8 bits are not taken", who);
    const int len = src->len;
    if (first < 0 || last < 0 || keep < 0 || (int64_t)first + last > keep) return fail(ANPD_E_INVAL, "%s: need 0 <= first + last <= keep", who);
    if (keep > len || keep > dst->max_tokens) return fail(ANPD_E_CAPACITY, "%s: %d positions of %d, into a cache of %d", who, keep, len, dst->max_tokens);
    if (!(rope_base == 0.f || rope_base > 1.f) || std::isinf(rope_base)) return fail(ANPD_E_INVAL, "%s: rope_base must be 0 or above 1", who);
    const int64_t heads = (int64_t)c.n_layers * c.n_kv_heads;
    if (keep > 0) {
        if (!mass || !out_kept) return fail(ANPD_E_INVAL, "%s: NULL argument", who);
        if (ld_mass < len || (out_mass && ld_out < keep)) return fail(ANPD_E_CAPACITY, "%s: rows of mass are shorter than their positions", who);
        if ((((uintptr_t)mass | (uintptr_t)out_kept | (uintptr_t)out_mass) & 3) != 0) return fail(ANPD_E_INVAL, "%s: an argument is not aligned to its type", who);
        const size_t mass_bytes = ((size_t)(heads - 1) * ld_mass + len) * sizeof(float), kept_bytes = (size_t)heads * keep * sizeof(int32_t);
        const size_t out_bytes = out_mass ? ((size_t)(heads - 1) * ld_out + keep) * sizeof(float) : 0;
        if (out_mass && overlap(mass, mass_bytes, out_mass, out_bytes)) return fail(ANPD_E_INVAL, "%s: out_mass overlaps mass", who);
        if (overlap(mass, mass_bytes, out_kept, kept_bytes) || (out_mass && overlap(out_mass, out_bytes, out_kept, kept_bytes)))
            return fail(ANPD_E_INVAL, "%s: out_kept overlaps mass or out_mass", who);
    }
    OnDevice on;
    int32_t rc = on.enter(who, src->device);
    if (rc != ANPD_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    if (keep > 0) {
        if ((rc = ensure_pages(dst, keep, st)) != ANPD_OK) return rc;
        SelectArgs a = {mass, out_kept, out_mass, ld_mass, ld_out, len, keep, first, last};
        const dim3 rows((unsigned)heads), threads(kSelectThreads);
        // positions per lane: as few registers as hold them
        if (len <= 4 * kSelectThreads) hipLaunchKernelGGL(cache_select_kernel<4>, rows, threads, 0, st, a);
        else if (len <= 16 * kSelectThreads) hipLaunchKernelGGL(cache_select_kernel<16>, rows, threads, 0, st, a);
        else if (len <= 64 * kSelectThreads) hipLaunchKernelGGL(cache_select_kernel<64>, rows, threads, 0, st, a);
        else hipLaunchKernelGGL(cache_select_kernel<0>, rows, threads, 0, st, a);
        HIP_TRY(hipGetLastError());
        MoveArgs m;
        std::memset(&m, 0, sizeof(m));
        m.src = src->pool;
        m.dst = dst->pool;
        m.src_table = src->d_table;
        m.dst_table = dst->d_table;
        m.dst_len = dst->d_len;
        m.kept = out_kept;
        m.rotate = rope_base > 0.f;
        m.keep = keep;
        m.n_layers = c.n_layers;
        m.n_kv_heads = c.n_kv_heads;
        m.page_tokens = c.page_tokens;
        for (int i = 0; i < c.head_dim / 2 && m.rotate; ++i) m.turn[i] = std::pow((double)rope_base, -2.0 * i / c.head_dim) / (2.0 * 3.14159265358979323846);
        const int groups = (keep + kMovePages * 16 - 1) / (kMovePages * 16);
        // (into itself a cache moves in order, by one block per layer, head and kind)
        const dim3 grid((unsigned)heads, 2, (unsigned)(dst == src ? 1 : groups));
#define ANPD_MOVE(KERNEL) hipLaunchKernelGGL((KERNEL), grid, dim3(kMoveThreads), 0, st, m)
        if (c.fragments) { if (c.head_dim == 128) ANPD_MOVE(cache_move_kernel<128>); else ANPD_MOVE(cache_move_kernel<64>); }
        else if (c.dtype == ANPD_BF16) {
            if (c.head_dim == 128) hipLaunchKernelGGL((cache_move_plain_kernel<bf16_t, 128>), grid, dim3(kMoveThreads), 0, st, m);
            else hipLaunchKernelGGL((cache_move_plain_kernel<bf16_t, 64>), grid, dim3(kMoveThreads), 0, st, m);
        } else if (c.head_dim == 128) hipLaunchKernelGGL((cache_move_plain_kernel<float, 128>), grid, dim3(kMoveThreads), 0, st, m);
        else hipLaunchKernelGGL((cache_move_plain_kernel<float, 64>), grid, dim3(kMoveThreads), 0, st, m);
#undef ANPD_MOVE
        HIP_TRY(hipGetLastError());
        HIP_TRY(hipStreamSynchronize(st));
        dst->len = keep;
        release_pages(dst, keep);
        return ANPD_OK;
    }
    return anpd_kv_truncate(dst, 0, stream);
}

}  // extern "C"
