// Attention over caches of 8-bit keys and values, for gfx950.
//
//   t_rj = scale s_j (q_r . c_j),   out_r = sum_j (p_rj s'_j) c'_j       c, c': codes of key and value; s, s': their scales
//
// Codes are whole numbers up to 127, which fp16 holds exactly, and one permutation and one packed sum make two of them operands: with bf16 they go through
// fp32, and one term of a weight is not enough (2^-8 of it, beside the output's own rounding; two terms: 32 tokens 41 us, not 38; 1001 fp32 rows 75, not 58).
// What fp16 lacks is range.  Rows are scaled by powers of two, so that their largest number is below 2^15 (numbers 2^29 below it are exact, others off by 2^-40 of it); rows of
// fp32 are two terms, 22 bits.  Weights carry their value's scale, p_rj s'_j, and a row's reference follows the largest of both, so that they are below 2^15: one term
// is within 2^-11 of a weight (where the output's own rounding to bf16 makes 2^-8), two within 2^-22.  A key whose values are 2^20 times smaller than those of another
// that the row sees begins to lose digits.
#pragma once
#include "anpd_cache_softmax.h"

namespace anpd {

// Launches the kernel below (a's blocks and splits as for blocks of 32 rows).
void launch_attention8(const AttnArgs &a, Seen rules, int head_dim, hipStream_t st);

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f16x8 as_f16(u32x4 v) { return __builtin_bit_cast(f16x8, v); }
__device__ __forceinline__ f32x16 mfma32h(f16x8 x, f16x8 y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0); }

// Eight bytes (codes + 128) as an operand: 0x6400 + byte is 1024 + byte in fp16.
__device__ __forceinline__ f16x8 codes8(uint32_t lo, uint32_t hi)
{
    u32x4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = __builtin_amdgcn_perm(0x64646464u, i < 2 ? lo : hi, i & 1 ? 0x04030402u : 0x04010400u);
        t[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, two) + (f16x2){(_Float16)-1152.0f, (_Float16)-1152.0f});
    }
    return as_f16(t);
}
// Eight numbers below 2^15 as TERMS fp16 operands that add up to them (rounded; within 22 bits).
template <int TERMS>
__device__ __forceinline__ void split_terms16(float (&x)[8], u32x4 (&t)[TERMS])
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
            const f16x2 h = __builtin_convertvector((f32x2){x[2 * i], x[2 * i + 1]}, f16x2);
            t[k][i] = __builtin_bit_cast(uint32_t, h);
            if (k + 1 < TERMS) { x[2 * i] -= (float)h[0]; x[2 * i + 1] -= (float)h[1]; }
        }
}
// The smallest scale of values that a reference follows.  An unscaled weight is below 2^15 divided by it, 2^107, and the sum of as many as a cache has positions, 2^20, below
// 2^127; with 2^-100, 2^17 keys whose values were zeros had an infinite sum.  Smaller scales lose digits from 2^-102 on (fp32 rows) or 2^-113 (bf16).
constexpr float kSmallestScale = 0x1p-93f;

// Block = (32 virtual rows, kv head, split of the keys), four waves; wave w takes keys 32 w .. of every 128, as in the form for bf16 pages.
// Tokens: 32 of 32 sequences of 300 to 700 positions, 140 MB in 35 us (4.0 TB/s): a block lives 14.5 us, of which start and end, that nothing overlaps but other
// blocks, are 7.7, so half the bytes are not half the time (bf16: 50).  One token behind 65535 positions of 8 key heads, 139 MB in 29 us (4.8 TB/s), joined in 4.
// Rows of prompts: the codes of every tile are made operands again for 32 rows (1001 fp32 rows of 32 heads 58 us; vector instructions 45 % of the
// cycles, matrix instructions 27 %).  Two waves a SIMD, as many as 256 registers allow; three spill (46 us instead of 38).
// grid: n_blocks * n_splits * n_kv_heads
template <int DH, int TERMS, int RULES>
__global__ __launch_bounds__(256, 2) void cache_attn8_kernel(const AttnArgs a)
{
    constexpr int NKS = DH / 16, NKC = DH / 32, NDT = DH / 32, NDB = DH / 64;
    __shared__ union {
        float part[kStreamWaves][2][16][64];
        u32x4 q[NKS][TERMS][64];   // the rows' terms
    } lds;
    __shared__ float wm[kStreamWaves][32], wl[kStreamWaves][32];
    __shared__ float scale_of[kStreamWaves][64];   // of the wave's 32 keys, then of their values
    __shared__ float most_of[kStreamWaves][32];     // largest of the rows' numbers that a wave has
    __shared__ int depth[RULES == kTree ? kTreeRows : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, m = lane & 31;
    const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int split = rest % a.n_splits, block = a.n_blocks - 1 - rest / a.n_splits;
    const SeqView s = a.seq[seq_of_block(a, block)];
    const int v0 = (block - s.block0) * kRowTile, total = s.pos0 + s.n;
    RowInfo r = row_info<RULES>(a, s, kvh, v0);
    const int pre = RULES && a.prefix > 0 ? (a.prefix < total ? a.prefix : total) : 0;
    const int p_lo = __builtin_amdgcn_readlane(r.p, 0), p_hi = __builtin_amdgcn_readlane(r.p, 31);
    const KeyTiles tiles = RULES == kTree ? key_tiles(s.pos0, total - 1, total, a.window, a.prefix, kStreamTile)
                                          : key_tiles(p_lo, p_hi, total, RULES ? a.window : 0, RULES ? a.prefix : 0, kStreamTile);
    const int begin = split * a.chunk, i1 = begin + a.chunk < tiles.n ? begin + a.chunk : tiles.n;
    if (begin >= tiles.n) return;   // (the whole block; what joins the splits does not look at this one)
    const int i0 = RULES ? first_tile(tiles, wave_min(r.fk), begin, i1, kStreamTile) : begin;   // (the same for all waves)

    Running<NDT> run;
    run.start();

    const int last_page = (total - 1) >> 4;
    const size_t page_bytes = (size_t)a.n_layers * 2 * a.n_kv_heads * kv8_block_bytes(DH);
    const char *k_of = (const char *)s.pool + ((size_t)a.layer * 2 * a.n_kv_heads + kvh) * kv8_block_bytes(DH), *v_of = k_of + (size_t)a.n_kv_heads * kv8_block_bytes(DH);
    // physical pages of the wave's next 64 tiles, a tile per lane (beyond the last key: the last page again)
    int ida = 0, idb = 0;
    auto fetch_ids = [&](int i) __attribute__((always_inline)) {
        const int t = i + lane < i1 ? i + lane : i1 - 1;
        const int page = tiles.at(t) * (kStreamTile / 16) + 2 * wave;
        ida = s.table[page < last_page ? page : last_page];
        idb = s.table[page + 1 < last_page ? page + 1 : last_page];
    };
    // Two tiles are on their way while a third is looked at: what 8 bits take of a compute unit's loads in flight would not keep the memory busy otherwise.
    u32x4 kf[2][NKC], vf[2][2][NDB];
    float scale[2];
    auto page_of = [&](int i, int which) __attribute__((always_inline)) { return (size_t)__builtin_amdgcn_readlane(which ? idb : ida, (i - i0) & 63) * page_bytes; };
    auto load_k = [&](int b, size_t pa, size_t pb) __attribute__((always_inline)) {
        const char *page = k_of + (lane & 16 ? pb : pa);
        const u32x4 *p = (const u32x4 *)page + half * 16 + (lane & 15);
#pragma unroll
        for (int x = 0; x < NKC; ++x) kf[b][x] = p[x * 32];
        scale[b] = *((const float *)(page + (half ? v_of - k_of : 0) + 16 * DH) + (lane & 15));
    };
    auto load_v = [&](int b, size_t pa, size_t pb) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const u32x4 *p = (const u32x4 *)(v_of + (g ? pb : pa)) + half * 32 + m;
#pragma unroll
            for (int d = 0; d < NDB; ++d) vf[b][g][d] = p[d * 64];
        }
    };
    if (i0 < i1) fetch_ids(i0);
    // What the first tiles' loads wait for (pages) and what is worked on behind them (the rows, the tree) is requested together.
    int up = -1;
    if constexpr (RULES == kTree) up = parent_of(a, s);
    float x[NKS / kStreamWaves][8];
#pragma unroll
    for (int y = 0; y < NKS / kStreamWaves; ++y) {
        const int ks = y * kStreamWaves + wave;
        load_q8(a, (size_t)r.row * a.ldq + (size_t)r.head * DH + 16 * half + 32 * (ks >> 1) + 8 * (ks & 1), x[y]);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (i0 < i1) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            load_k(b, page_of(i0 + b, 0), page_of(i0 + b, 1));
            __builtin_amdgcn_sched_barrier(0);   // (in the loop's order, or its waits would be for what comes last here)
            load_v(b, page_of(i0 + b, 0), page_of(i0 + b, 1));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (RULES == kTree) tree_info(a, s, pre, up, depth, r);
    // The rows' terms.  A step of 16 dims: 8 y .. of the 16 that a half of the wave has of every 32.
    float row_scale;
    {
        float most = 0.f;
        bool finite = true;
#pragma unroll
        for (int y = 0; y < NKS / kStreamWaves; ++y)
#pragma unroll
            for (int e = 0; e < 8; ++e) { most = fmaxf(most, fabsf(x[y][e])); finite = finite && fabsf(x[y][e]) <= 3.4028234e38f; }
        most = both_halves_max(finite ? most : INFINITY);
        if (half == 0) most_of[wave][m] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kStreamWaves; ++w) most = fmaxf(most, most_of[w][m]);
        int by = most > 0.f && most < INFINITY ? 15 - __builtin_amdgcn_frexp_expf(most) : 0;
        by = by < 100 ? by : 100;   // (what is smaller has scores of 0)
        row_scale = ldexpf(1.0f, -by);
#pragma unroll
        for (int y = 0; y < NKS / kStreamWaves; ++y) {
            u32x4 q[TERMS];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[y][e] = most < INFINITY ? ldexpf(x[y][e], by) : __uint_as_float(0x7fc00000u);   // (a row with an infinity or a NaN: NaN, where it sees a key)
            split_terms16<TERMS>(x[y], q);
#pragma unroll
            for (int t = 0; t < TERMS; ++t) lds.q[y * kStreamWaves + wave][t][lane] = q[t];
        }
        __syncthreads();
    }
    // Products to exponents: in the factor, or where the rules change the scores, in the products themselves.
    constexpr Scored HOW = !RULES ? kUnscored : TERMS == 1 ? kScoredRough : kScored;
    const bool scored = HOW != kUnscored && (a.cap > 0.f || a.slopes);   // (the same for all)
    const float factor = scored ? score_factor<HOW>(a) : score_factor<HOW>(a) * row_scale;
    auto tile = [&](int i, int b) __attribute__((always_inline)) {
        const int base = tiles.at(i) * kStreamTile + 32 * wave;
        if (((i + 2 - i0) & 63) == 0) {
            fetch_ids(i + 2);
            asm volatile("" : "+v"(ida), "+v"(idb));   // (waited for here: in front of their use all loads in flight would be, at every tile)
        }
        const size_t na = page_of(i + 2, 0), nb = page_of(i + 2, 1);
        __builtin_amdgcn_wave_barrier();
        scale_of[wave][lane] = scale[b];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        f32x16 sc[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[0][e] = 0.f;
        int at = lane;
        asm volatile("" : "+v"(at));   // (read anew for each tile)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            const f16x8 k = codes8(kf[b][ks >> 1][2 * (ks & 1)], kf[b][ks >> 1][2 * (ks & 1) + 1]);
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t) sc[0] = mfma32h(k, as_f16(lds.q[ks][t][at]), sc[0]);
        }
        load_k(b, na, nb);
        if (i < i1 && any_seen<RULES>(r, pre, base)) {
            f32x4 value_scale[4];
            float largest = kSmallestScale;
            const bool hidden = !all_seen<RULES>(r, pre, base);
            const SeenOf<RULES> seen(r, pre, base);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                f32x4 x = *(const f32x4 *)&scale_of[wave][2 * e + 4 * half], y = *(const f32x4 *)&scale_of[wave][32 + 2 * e + 4 * half];
                if (scored) x = x * row_scale;
#pragma unroll
                for (int u = 0; u < 4; ++u) sc[0][e + u] *= x[u];
                if (hidden) {   // (a scale that is NaN must not meet a weight of 0, nor one that is not seen raise the reference)
#pragma unroll
                    for (int u = 0; u < 4; ++u) y[u] = seen[e + u] ? y[u] : 0.f;
                }
                value_scale[e >> 2] = y;
                largest = fmaxf(fmaxf(largest, fmaxf(y[0], y[1])), fmaxf(y[2], y[3]));
            }
            finish_scores<RULES, HOW, 1>(a, r, pre, base, sc);
            // The reference: weights are below 2^15, and when it moves, the largest so far is between 2^6 and 2^7 if the largest score's values are the largest.
            float most = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; e += 2) most = fmaxf(fmaxf(most, sc[0][e]), sc[0][e + 1]);
            most = both_halves_max(most) * factor + (float)__builtin_amdgcn_frexp_expf(both_halves_max(largest));
            move_reference(run, most > run.m + 15.f ? most - 7.f : run.m);
            run.l += huge_reference(run.m) ? careful_weights<1>(sc, factor, run.m) : weights<1>(sc, factor, run.m);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sc[0][8 * g + e] * value_scale[2 * g + (e >> 2)][e & 3];
                u32x4 w[TERMS];
                split_terms16<TERMS>(x, w);
#pragma unroll
                for (int d = 0; d < NDT; ++d) {
                    const int odd = 2 * (d & 1);
                    const f16x8 v = codes8(vf[b][g][d >> 1][odd], vf[b][g][d >> 1][odd + 1]);
#pragma unroll
                    for (int t = TERMS - 1; t >= 0; --t) run.o[d] = mfma32h(v, as_f16(w[t]), run.o[d]);
                }
            }
        }
        load_v(b, na, nb);
    };
    if (i0 < i1) {
        // (one exit, and the same loads on every way through the loop, behind the last tile for nothing: otherwise they could not be counted)
        for (int i = i0; i < i1; i += 2) {
            tile(i, 0);
            tile(i + 1, 1);
        }
    }
    waves_meet<DH>(a, r, block, kvh, split, tiles.n, run, lds.part, wm, wl);
}

}  // namespace anpd
