// What attention over paged caches is made of: rows and the keys they see, operands, the running softmax, results (gfx950).
//
//   t_rj = scale q_r . k_j,   cap > 0: t = cap tanh(t / cap),   t -= slope_h |p_r - j|
//   out_r = sum_j exp(t_rj - lse_r) v_j,   lse_r = log sum_j exp t_rj        over the keys that row r sees
// where j is a key's position: its slot in the cache, or in a tree of new rows the number of the cached positions and of its ancestors
//   mass_gj += sum over the rows r and query heads h of group g of exp(t_rj - lse_r)
//
// Rows.  The query heads that share a key / value head read the same keys, so they are rows of one matrix: "virtual row"
// v = r * group + h stands for head h of the group in row r.  Keys are then read once for all of them, and a token of a
// model with 16 query heads per key / value head is 16 rows of a matrix product and not 16 products of one row.
//
// Products.  S^T = K q^T with 32x32 matrix instructions: a lane has 16 keys (8 (i / 4) + 4 half + i % 4, half = lane / 32) of
// ONE row (lane % 32), so a row's maximum and sum are in-lane but for one exchange of the wave's halves, and the weights are,
// as they stand in registers, the operand of O^T += V^T P: two groups of four keys per 16-key page and half.  The cache's
// fragment order has both operands ready: K in 16-byte pieces of 8 dims of a key, V in 8-byte pieces of 4 keys of a dim.
//
// Precision.  Scores, maxima, sums and outputs are held in 32 bits.  bf16 rows meet bf16 keys exactly; their weights are
// rounded to bf16 for the second product (2^-8 of a weight at most, as the output's own rounding).  fp32 rows are three bf16
// terms, 24 bits, and so are their weights: two terms lose up to 2^-16 of every weight, which was ten times the error of fp32 sums.
#pragma once
#include <type_traits>

#include "anpd_layout.h"

namespace anpd {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttnMaxSeqs = ANPD_ATTN_MAX_SEQS;
constexpr int kRowTile = 32;              // virtual rows of a wave
constexpr float kNoKey = -3.0e38f;        // a row's reference before it has seen a key
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

struct SeqView {
    const void *pool;
    const int32_t *table;   // physical pages
    int32_t pos0, n, row0;  // position of the first new row, new rows, the first one's place among the rows of all sequences
    int32_t block0;         // first row block
};

struct AttnArgs {
    SeqView seq[kAttnMaxSeqs];
    const void *q;
    void *out;
    float *lse;                 // [rows][heads]; may be NULL in attention
    const float *slopes;        // [heads] or NULL
    const int32_t *first_key;   // [rows] or NULL
    const int32_t *parent;      // [rows]: the new rows of every sequence are a tree (kTree); otherwise NULL
    float *part;                // attention: partial results of splits, or NULL; mass: partial sums, or NULL
    int64_t ldq, ldo;           // elements between rows
    float scale, cap, scale_over_cap;
    int32_t window, prefix;     // 0: none
    int32_t layer, n_layers, n_heads, n_kv_heads, group, page_tokens;
    int32_t q_f32, q_wide;      // type of the rows and outputs; whether rows and outputs may be moved 16 bytes at a time
    int32_t n_seq, n_blocks, n_splits, chunk;   // row blocks of all sequences; splits of the keys, tiles in each
};

struct MassOut {
    float *mass[kAttnMaxSeqs];   // [kv head][ld]
    int64_t ld;
};

// ------------------------------------------------------------------ rows and their keys

// Which keys a row sees: all up to its own, those that the rules leave, or, where the new rows are a tree, those of the cached ones that
// the rules leave and of the new ones its ancestors and itself.
enum Seen { kCausal, kRuled, kTree };
constexpr int kTreeRows = ANPD_TREE_MAX_ROWS;   // a bit each

// What a lane knows of its row.
struct RowInfo {
    int v;        // virtual row of the sequence (the last one again for lanes beyond it)
    int row, head;   // its row among those of all sequences, its query head
    int p;        // position
    int fk, lo;   // first visible key; the same with the window
    float slope;
    bool live;    // a row of its own
    int cached;                  // trees: positions in front of the new rows,
    unsigned long long chain;    // which of these the row sees, a bit each,
    const int *depth;            // and how many ancestors each of them has
};
// (a number below 0 is 0: differences of it and positions stay in 32 bits)
__device__ __forceinline__ int first_key_of(const AttnArgs &a, int row)
{
    const int fk = a.first_key ? a.first_key[row] : 0;
    return fk > 0 ? fk : 0;
}
template <int RULES>
__device__ __forceinline__ RowInfo row_info(const AttnArgs &a, const SeqView &s, int kvh, int v0)
{
    const int total = s.n * a.group, v = v0 + (threadIdx.x & 31);
    RowInfo r;
    r.live = v < total;
    r.v = r.live ? v : total - 1;
    r.row = r.v / a.group;
    r.head = kvh * a.group + (r.v - r.row * a.group);
    r.p = s.pos0 + r.row;
    r.row += s.row0;
    r.fk = 0;
    r.lo = 0;
    r.slope = 0.f;
    if (RULES) {
        if (a.slopes) r.slope = a.slopes[r.head];
        r.fk = first_key_of(a, r.row);
        r.lo = r.fk;
        if (a.window > 0) { const int lo = r.p - a.window + 1; r.lo = lo > r.fk ? lo : r.fk; }
    }
    return r;
}

__device__ __forceinline__ unsigned long long shuffle64(unsigned long long v, int from)
{
    return ((unsigned long long)(uint32_t)__shfl((int)(v >> 32), from, 64) << 32) | (uint32_t)__shfl((int)v, from, 64);
}
// A chain without its lowest `count` bits.
__device__ __forceinline__ unsigned long long from_position(unsigned long long chain, int count)
{
    for (; count > 0 && chain != 0; --count) chain &= chain - 1;
    return chain;
}
// The tree of a sequence's new rows, for the lane's row.  Lane l looks at new row l: in step i it has the nearest 2^i of its ancestors, and takes over
// those of the last one of them: six steps, the same for every wave (32 heads of 128, captured: a tree of 8 behind 128 positions 7.6 us, where 8 rows that follow
// one another take 6.4; of 32 behind 2048 14.5 and 13.3).  A parent that is not an earlier row is none: the row follows the cached positions.  up: what
// parent_of says, requested before; depth: LDS, kTreeRows numbers, the same from every wave that writes them.
__device__ __forceinline__ int parent_of(const AttnArgs &a, const SeqView &s) { return (int)(threadIdx.x & 63) < s.n ? a.parent[s.row0 + (threadIdx.x & 63)] : -1; }
__device__ __forceinline__ void tree_info(const AttnArgs &a, const SeqView &s, int pre, int up, int *depth, RowInfo &r)
{
    const int lane = threadIdx.x & 63;
    if (up < 0 || up >= lane) up = -1;
    unsigned long long chain = 1ull << lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const int from = up < 0 ? lane : up;
        const unsigned long long c = shuffle64(chain, from);
        const int u = __shfl(up, from, 64);
        if (up >= 0) { chain |= c; up = u; }
    }
    const int d = __popcll(chain) - 1;
    depth[lane] = d;
    if (a.window > 0 || a.first_key) {
        // By positions, as for cached keys: bits of a chain ascend with their positions pos0, pos0 + 1, ..., so what lies before a position are its lowest ones.
        const int fk = lane < s.n ? first_key_of(a, s.row0 + lane) : 0, at = s.pos0 + d, lo = a.window > 0 && at - a.window + 1 > fk ? at - a.window + 1 : fk;
        const unsigned long long late = from_position(chain, lo - s.pos0);
        const unsigned long long early = pre > s.pos0 && fk < pre ? from_position(chain, fk - s.pos0) & ~from_position(chain, pre - s.pos0) : 0;
        chain = late | early;
    }
    const int row = r.row - s.row0;
    r.chain = shuffle64(chain, row);
    r.p = s.pos0 + __shfl(d, row, 64);
    r.cached = s.pos0;
    r.depth = depth;
    if (a.window > 0) { const int lo = r.p - a.window + 1; r.lo = lo > r.fk ? lo : r.fk; }
}
// Position of the key in slot j.
template <int RULES>
__device__ __forceinline__ int position_of(const RowInfo &r, int j)
{
    return RULES == kTree && j >= r.cached ? r.cached + r.depth[(j - r.cached) & (kTreeRows - 1)] : j;
}

// Which of the 32 keys from `base` on a row sees, a bit each.
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
template <int RULES>
__device__ __forceinline__ uint32_t seen_bits(const RowInfo &r, int pre, int base)
{
    const int o = base - r.cached, end = RULES == kTree ? r.cached : r.p + 1;
    const uint32_t late = below(end - base) & ~below(r.lo - base), early = below((RULES == kTree && pre > end ? end : pre) - base) & ~below(r.fk - base);
    if (RULES != kTree) return late | early;
    return late | early | (o >= kTreeRows || o <= -32 ? 0u : (uint32_t)(o >= 0 ? r.chain >> o : r.chain << -o));
}
template <int RULES>
__device__ __forceinline__ bool sees(const RowInfo &r, int pre, int j)
{
    if (RULES == kTree) return j < r.cached ? j >= r.lo || (j < pre && j >= r.fk) : j - r.cached < kTreeRows && (r.chain >> (j - r.cached) & 1);
    return RULES ? (j <= r.p && j >= r.lo) || (j < pre && j >= r.fk) : j <= r.p;
}
// Whether the lane's row sees key 8 (i / 4) + 4 half + i % 4 of the 32 from `base` on, as a product's element i.  Rules are a word of bits, formed once for
// a tile: with four comparisons for each key, or shifts of 64 bits for a tree, 3584 rows in documents of 500 took 78 us instead of 66, a tree of 8 behind 128
// positions 8.8 instead of 7.6.
template <int RULES>
struct SeenOf {
    const RowInfo &r;
    int pre, base;
    uint32_t word;
    __device__ __forceinline__ SeenOf(const RowInfo &row, int prefix, int from) : r(row), pre(prefix), base(from + 4 * ((threadIdx.x >> 5) & 1)), word(0)
    {
        if (RULES) {
            word = seen_bits<RULES>(row, prefix, from) >> (4 * ((threadIdx.x >> 5) & 1));
            asm volatile("" : "+v"(word));   // (bits of it, not sixteen conditions, are kept)
        }
    }
    __device__ __forceinline__ bool operator[](int i) const
    {
        if (RULES) return word & 1u << (8 * (i >> 2) + (i & 3));
        return sees<RULES>(r, pre, base + 8 * (i >> 2) + (i & 3));
    }
};
// Of the 32 keys from `base` on: does any of the wave's rows see one, do all see all?
template <int RULES>
__device__ __forceinline__ bool any_seen(const RowInfo &r, int pre, int base)
{
    if (RULES == kTree) {
        if (base + 31 < r.cached) return __builtin_amdgcn_ballot_w64(base + 31 >= r.lo || (base < pre && base + 31 >= r.fk)) != 0;
        return __builtin_amdgcn_ballot_w64(seen_bits<RULES>(r, pre, base) != 0) != 0;
    }
    return __builtin_amdgcn_ballot_w64(RULES ? (base <= r.p && base + 31 >= r.lo && r.lo <= r.p) || (base < pre && base + 31 >= r.fk) : base <= r.p) != 0;
}
template <int RULES>
__device__ __forceinline__ bool all_seen(const RowInfo &r, int pre, int base)
{
    if (RULES == kTree) return base + 31 < r.cached && __builtin_amdgcn_ballot_w64(!(base >= r.lo || (base + 31 < pre && base >= r.fk))) == 0;
    return __builtin_amdgcn_ballot_w64(!(RULES ? (base + 31 <= r.p && base >= r.lo) || (base + 31 < pre && base >= r.fk) : base + 31 <= r.p)) == 0;
}

// The key tiles (of `tile` keys) that rows with positions p_lo .. p_hi can see: the prefix, then what the window leaves.
// Known on the host as well (first_key is not looked at).
struct KeyTiles {
    int a, b0, n;   // tiles of the prefix; the first one behind them that is visited; how many are visited
    __host__ __device__ int at(int i) const { return i < a ? i : b0 + (i - a); }
};
__host__ __device__ __forceinline__ KeyTiles key_tiles(int p_lo, int p_hi, int total, int window, int prefix, int tile)
{
    KeyTiles k;
    const int pre = prefix < total ? prefix : total;
    const int lo = window > 0 && p_lo - window + 1 > 0 ? p_lo - window + 1 : 0;
    k.a = (pre + tile - 1) / tile;
    k.b0 = lo / tile > k.a ? lo / tile : k.a;
    const int b1 = p_hi / tile + 1;
    k.n = k.a + (b1 > k.b0 ? b1 - k.b0 : 0);
    return k;
}

// ... of the rows at p_lo .. p_hi of a sequence, in a tree of any (the lowest position is the first, the last key the last slot)
__host__ __device__ __forceinline__ KeyTiles key_tiles(const AttnArgs &a, const SeqView &s, int p_lo, int p_hi, int tile)
{
    const int total = s.pos0 + s.n;
    return a.parent ? key_tiles(s.pos0, total - 1, total, a.window, a.prefix, tile) : key_tiles(p_lo, p_hi, total, a.window, a.prefix, tile);
}

__device__ __forceinline__ int wave_min(int v)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) { const int w = __shfl_xor(v, o, 64); v = w < v ? w : v; }
    return __builtin_amdgcn_readfirstlane(v);
}
// The first of tiles i0 .. i1 - 1 that does not lie wholly below key fk (i1: none); tiles are in the order of their keys.
__device__ __forceinline__ int first_tile(const KeyTiles &k, int fk, int i0, int i1, int tile)
{
    if (fk <= 0) return i0;
    const int t = fk / tile, i = t <= k.a ? t : (t <= k.b0 ? k.a : k.a + (t - k.b0));
    return i < i0 ? i0 : (i < i1 ? i : i1);
}

// For cap tanh(t / cap): 1 - 2 / (1 + e^2x) is off by 2^-22 at most, whatever x is, which is nothing beside weights in bf16 unless the cap
// is large (ROUGH: caps up to kRoughCap, 2^-14 of a score); otherwise small x take a sum of powers, to 2^-23 of the value.
constexpr float kRoughCap = 256.f;
template <bool ROUGH>
__device__ __forceinline__ float tanh_f32(float x)
{
    const float t = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * (2.0f * kLog2e))), 1.0f);
    if (ROUGH) return t;
    const float y = x * x;
    float s = fmaf(y, -1382.0f / 155925.0f, 62.0f / 2835.0f);
    s = fmaf(y, s, -17.0f / 315.0f);
    s = fmaf(y, s, 2.0f / 15.0f);
    s = fmaf(y, s, -1.0f / 3.0f);
    s = fmaf(y * x, s, x);
    return y < 0.08f ? s : t;
}

// Products to scores where there are rules (cap, bias): natural units.
template <bool ROUGH>
__device__ __forceinline__ float ruled_score(const AttnArgs &a, float product, float slope, int distance)
{
    float t = a.cap > 0.f ? a.cap * tanh_f32<ROUGH>(product * a.scale_over_cap) : product * a.scale;
    if (a.slopes) t = fmaf(-slope, (float)(distance < 0 ? -distance : distance), t);
    return t;
}

// ------------------------------------------------------------------ operands

__device__ __forceinline__ bf16x8 as_bf16(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ f32x16 mfma32(bf16x8 x, bf16x8 y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0); }

// Two numbers as words of TERMS bf16 operands.
template <int TERMS>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&t)[TERMS])
{
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
        t[k] = pack_bf16(x, y);
        if (k + 1 < TERMS) {
            x -= __uint_as_float(t[k] << 16);
            y -= __uint_as_float(t[k] & 0xffff0000u);
        }
    }
}
// Eight numbers as TERMS bf16 operands that add up to them (1: rounded; 3: exact but for the smallest of numbers).
template <int TERMS>
__device__ __forceinline__ void split_terms(const float (&x)[8], u32x4 (&t)[TERMS])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t w[TERMS];
        split_pair<TERMS>(x[2 * i], x[2 * i + 1], w);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) t[k][i] = w[k];
    }
}

// Eight dims of a row, whatever its type and alignment.
__device__ __forceinline__ void load_q8(const AttnArgs &a, size_t at, float (&x)[8])
{
    if (a.q_f32) {
        const float *p = (const float *)a.q + at;
        if (a.q_wide) {
            const f32x4 u = *(const f32x4 *)p, v = *(const f32x4 *)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
    } else {
        const bf16_t *p = (const bf16_t *)a.q + at;
        if (a.q_wide) {
            const u32x4 u = *(const u32x4 *)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(p[i]);
        }
    }
}
template <int TERMS>
__device__ __forceinline__ void load_q8(const AttnArgs &a, size_t at, u32x4 (&t)[TERMS])
{
    if constexpr (TERMS == 1) {   // (bf16 rows are the operand as they are)
        const bf16_t *p = (const bf16_t *)a.q + at;
        if (a.q_wide) t[0] = *(const u32x4 *)p;
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) t[0][i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
        }
    } else {
        float x[8];
        load_q8(a, at, x);
        split_terms<TERMS>(x, t);
    }
}
// ------------------------------------------------------------------ the running softmax of a wave's rows

// A lane's numbers: the row's reference (base 2), the sum of its own half's weights, the output's 16 dims per tile of 32.
template <int NDT>
struct Running {
    float m, l;
    f32x16 o[NDT];
    __device__ __forceinline__ void start()
    {
        m = kNoKey;
        l = 0.f;
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
};

__device__ __forceinline__ float both_halves_max(float v)
{
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float both_halves_sum(float v)
{
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

// How the rules change the scores themselves (cap, bias): not at all, to what bf16 weights are worth where that will do, or in full.
enum Scored { kUnscored, kScoredRough, kScored };
// What is multiplied with a score to have its exponent in base 2.
template <Scored HOW>
__device__ __forceinline__ float score_factor(const AttnArgs &a)
{
    return HOW != kUnscored && (a.cap > 0.f || a.slopes) ? kLog2e : a.scale * kLog2e;
}
// Products of NB x 32 keys -> scores: the rules, and minus infinity for the keys that the row does not see.
template <int RULES, Scored HOW, int NB>
__device__ __forceinline__ void finish_scores(const AttnArgs &a, const RowInfo &r, int pre, int base, f32x16 (&s)[NB])
{
    const int half = (threadIdx.x >> 5) & 1;
    if (HOW != kUnscored && (a.cap > 0.f || a.slopes)) {   // (the same for all)
        if (HOW == kScoredRough && a.cap <= kRoughCap) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = ruled_score<true>(a, s[b][i], r.slope, r.p - position_of<RULES>(r, base + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3)));
        } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = ruled_score<false>(a, s[b][i], r.slope, r.p - position_of<RULES>(r, base + 32 * b + 8 * (i >> 2) + 4 * half + (i & 3)));
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if (all_seen<RULES>(r, pre, base + 32 * b)) continue;   // (the same for the whole wave)
        const SeenOf<RULES> seen(r, pre, base + 32 * b);
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (!seen[i]) s[b][i] = -INFINITY;
    }
}
// The row's reference with these scores: it follows the row's maximum only when that is more than 2^8 above it.  Weights are at most 2^8
// then, which costs no precision, and the output is rescaled a few times instead of at every other tile.
template <int NB>
__device__ __forceinline__ float new_reference(const f32x16 (&s)[NB], float factor, float m)
{
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[b][i]), s[b][i + 1]);
    mx = both_halves_max(mx) * factor;
    return mx > m + 8.f ? mx : m;
}
// Sum and output, which hold all weights formed so far, are moved to the new reference.
template <int NDT>
__device__ __forceinline__ void move_reference(Running<NDT> &run, float m_new)
{
    const float alpha = __builtin_amdgcn_exp2f(run.m - m_new);
    run.m = m_new;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f) == 0) return;   // (a factor of 1 changes nothing)
    run.l *= alpha;
#pragma unroll
    for (int d = 0; d < NDT; ++d) run.o[d] = run.o[d] * alpha;
}
// Where a reference is huge, the fused product is not the product that it was rounded from, and the difference, up to 2^-24 of it, would
// be the largest key's exponent: careful_weights then.  (The same for the whole wave.)
__device__ __forceinline__ bool huge_reference(float m) { return __builtin_amdgcn_ballot_w64(fabsf(m) > 0x1p28f) != 0; }
__device__ __forceinline__ float sum16(const f32x16 &s)
{
    float t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = (s[4 * i] + s[4 * i + 1]) + (s[4 * i + 2] + s[4 * i + 3]);
    return (t[0] + t[1]) + (t[2] + t[3]);
}
// Scores -> weights, in place, and their sum.
template <int NB>
__device__ __forceinline__ float weights(f32x16 (&s)[NB], float factor, float m)
{
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], factor, -m));
    float sum = sum16(s[0]);
#pragma unroll
    for (int b = 1; b < NB; ++b) sum += sum16(s[b]);
    return sum;
}
template <int NB>
__device__ __forceinline__ float careful_weights(f32x16 (&s)[NB], float factor, float m)
{
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float t = s[b][i] * factor;
            asm volatile("" : "+v"(t));   // (rounded here)
            s[b][i] = __builtin_amdgcn_exp2f(t - m);
        }
    float sum = sum16(s[0]);
#pragma unroll
    for (int b = 1; b < NB; ++b) sum += sum16(s[b]);
    return sum;
}
// All of it, one step after the other.
template <int RULES, Scored HOW, int NB, int NDT>
__device__ __forceinline__ void weigh(const AttnArgs &a, const RowInfo &r, int pre, int base, f32x16 (&s)[NB], Running<NDT> &run)
{
    const float factor = score_factor<HOW>(a);
    finish_scores<RULES, HOW, NB>(a, r, pre, base, s);
    move_reference(run, new_reference<NB>(s, factor, run.m));
    run.l += huge_reference(run.m) ? careful_weights<NB>(s, factor, run.m) : weights<NB>(s, factor, run.m);
}

// Where some key of a tile is hidden from some row, its values must not meet a weight of 0 if they are infinite or NaN: that product
// is NaN.  Such values are taken out of the tile (the return value says that there were any), and once the wave's tiles are through, added
// to the outputs of the rows that see them, which are infinite or NaN from then on whatever else there is.
template <int N>
__device__ __forceinline__ bool take_out_unbounded(u32x4 (&v)[N])
{
    uint32_t found = 0;   // exponents of all ones, as carries out of them
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) found |= ((v[n][i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
    if (__builtin_amdgcn_ballot_w64(found != 0) == 0) return false;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w = v[n][i];
            v[n][i] = ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
        }
    return true;
}
// The 32 keys from `base` on: value(j, dim) of key j, dim(d, i) of the lane's outputs.
template <int RULES, int NDT, typename Dim, typename Value>
__device__ __forceinline__ void add_unbounded(const RowInfo &r, int pre, int base, Running<NDT> &run, Dim dim, Value value)
{
    for (int j = base; j < base + 32; ++j) {
        if (!sees<RULES>(r, pre, j)) continue;
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float v = value(j, dim(d, i));
                if (!(fabsf(v) <= 3.4028234e38f)) run.o[d][i] += v;
                if (i % 4 == 3) asm volatile("" ::: "memory");   // (four at a time: this is no place for registers)
            }
    }
}

// ------------------------------------------------------------------ results

// Four adjacent dims of a row.
__device__ __forceinline__ void store_out4(const AttnArgs &a, int head_dim, int row, int head, int dim, f32x4 x)
{
    const size_t at = (size_t)row * a.ldo + (size_t)head * head_dim + dim;
    if (a.q_f32) {
        float *p = (float *)a.out + at;
        if (a.q_wide) *(f32x4 *)p = x;
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = x[i];
        }
    } else {
        bf16_t *p = (bf16_t *)a.out + at;
        const uint2 w = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        if (a.q_wide) *(uint2 *)p = w;
        else {
            p[0] = (bf16_t)w.x; p[1] = (bf16_t)(w.x >> 16); p[2] = (bf16_t)w.y; p[3] = (bf16_t)(w.y >> 16);
        }
    }
}
__device__ __forceinline__ void store_lse(const AttnArgs &a, int row, int head, float m, float l)
{
    // (a row without a key: -infinity)
    if (a.lse) a.lse[(size_t)row * a.n_heads + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : 1.0f / l; }

// Where a split's results lie: per (row block, kv head, split) [row][dim] and then [row] of (reference, sum).
__host__ __device__ __forceinline__ size_t part_floats(int rows, int head_dim) { return (size_t)rows * (head_dim + 2); }

// The sequence of a row block (the last one whose blocks begin at or before it; sequences without rows have none).
__device__ __forceinline__ int seq_of_block(const AttnArgs &a, int block)
{
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.seq[mid].block0 <= block) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

constexpr int kStreamWaves = 4, kStreamTile = 32 * kStreamWaves;   // of the forms of few rows: a wave takes 32 keys of every 128

// The waves of a block with results for the same 32 rows meet: every wave scales to the row's reference, the sums are formed in wave order.  Outputs are two
// tiles side by side: lane m of tile d has dims 64 (d / 2) + 2 (8 (i / 4) + 4 half + i % 4) + d % 2.
template <int DH>
__device__ __forceinline__ void waves_meet(const AttnArgs &a, const RowInfo &r, int block, int kvh, int split, int n_tiles, const Running<DH / 32> &run,
                                           float (&part)[kStreamWaves][2][16][64], float (&wm)[kStreamWaves][32], float (&wl)[kStreamWaves][32])
{
    constexpr int NDB = DH / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, m = lane & 31;
    const float l = both_halves_sum(run.l);
    if (half == 0) { wm[wave][m] = run.m; wl[wave][m] = l; }
    __syncthreads();
    float top = wm[0][m];
#pragma unroll
    for (int w = 1; w < kStreamWaves; ++w) top = fmaxf(top, wm[w][m]);
    const float f = __builtin_amdgcn_exp2f(run.m - top);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kStreamWaves; ++w) sum = fmaf(wl[w][m], __builtin_amdgcn_exp2f(wm[w][m] - top), sum);
    float *to = a.part && n_tiles > a.chunk ? a.part + (((size_t)block * a.n_kv_heads + kvh) * a.n_splits + split) * part_floats(kRowTile, DH) : nullptr;
    if (wave == 0 && half == 0 && r.live) {   // (beyond the last row nobody asks)
        if (to) *(float2 *)(to + kRowTile * DH + 2 * m) = make_float2(top, sum);
        else store_lse(a, r.row, r.head, top, sum);
    }
    const float inv = inverse_sum(sum);
#pragma unroll
    for (int d = 0; d < NDB; ++d) {
        if (d > 0) __syncthreads();
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const f32x16 o = run.o[2 * d + odd] * f;
#pragma unroll
            for (int i = 0; i < 16; ++i) part[wave][odd][i][lane] = o[i];
        }
        __syncthreads();
        // wave w finishes registers 4 w .. 4 w + 3 of both tiles: eight adjacent dims of the lane's row
        f32x4 x[2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                float t = part[0][odd][4 * wave + i][lane];
#pragma unroll
                for (int w = 1; w < kStreamWaves; ++w) t += part[w][odd][4 * wave + i][lane];
                x[i >> 1][2 * (i & 1) + odd] = t;
            }
        const int dim = 64 * d + 16 * wave + 8 * half;
        if (!r.live) continue;
        if (to) {
            *(f32x4 *)(to + m * DH + dim) = x[0];
            *(f32x4 *)(to + m * DH + dim + 4) = x[1];
        } else {
            store_out4(a, DH, r.row, r.head, dim, x[0] * inv);
            store_out4(a, DH, r.row, r.head, dim + 4, x[1] * inv);
        }
    }
}

}  // namespace anpd
