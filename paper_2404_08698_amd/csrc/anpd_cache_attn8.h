// Attention over caches of 8-bit keys and values, for gfx950.
//
//   t_rj = scale s_j (q_r . c_j),   out_r = sum_j (p_rj s'_j) c'_j       c, c': codes of key and value; s, s': their scales
//
// Codes are whole numbers of 7 bits and a sign, which bf16 holds exactly: they meet the same products as bf16 keys and values do, and the scales
// are applied to what a lane has of its row, scores and weights, in 32 bits.
#pragma once
#include "anpd_cache_softmax.h"

namespace anpd {

// Launches the kernel below (a's blocks and splits as for blocks of 32 rows).
void launch_attention8(const AttnArgs &a, Seen rules, int head_dim, hipStream_t st);

// Eight codes as an operand.
__device__ __forceinline__ u32x4 codes8(uint32_t lo, uint32_t hi)
{
    u32x4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? lo : hi;
        const float x = (float)(int8_t)(w >> (16 * (i & 1))), y = (float)(int8_t)(w >> (16 * (i & 1) + 8));
        t[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);   // (the lower halves are zero)
    }
    return t;
}

// Block = (32 virtual rows, kv head, split of the keys), four waves; wave w takes keys 32 w .. of every 128, as in the form for bf16 pages.
// grid: n_blocks * n_splits * n_kv_heads
template <int DH, int TERMS, int RULES>
__global__ __launch_bounds__(256, 2) void cache_attn8_kernel(const AttnArgs a)
{
    constexpr int NKS = DH / 16, NKC = DH / 32, NDT = DH / 32, NDB = DH / 64;
    constexpr bool SHARED_Q = TERMS > 1;   // (the rows' terms in LDS)
    __shared__ union {
        float part[kStreamWaves][2][16][64];
        u32x4 q[SHARED_Q ? NKS : 1][TERMS][64];
    } lds;
    __shared__ float wm[kStreamWaves][32], wl[kStreamWaves][32];
    __shared__ float scale_of[kStreamWaves][64];   // of the wave's 32 keys, then of their values
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
    if constexpr (RULES == kTree) tree_info(a, s, pre, depth, r);

    // A step of 16 dims: 8 y .. of the 16 that a half of the wave has of every 32.
    u32x4 q[SHARED_Q ? 1 : NKS][TERMS];
    {
        const size_t at = (size_t)r.row * a.ldq + (size_t)r.head * DH + 16 * half;
        if (SHARED_Q) {
#pragma unroll
            for (int x = 0; x < NKS / kStreamWaves; ++x) {
                const int ks = x * kStreamWaves + wave;
                load_q8<TERMS>(a, at + 32 * (ks >> 1) + 8 * (ks & 1), q[0]);
#pragma unroll
                for (int t = 0; t < TERMS; ++t) lds.q[ks][t][lane] = q[0][t];
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int ks = 0; ks < (SHARED_Q ? 1 : NKS); ++ks) load_q8<TERMS>(a, at + 32 * (ks >> 1) + 8 * (ks & 1), q[ks]);
        }
    }
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
    u32x4 kf[NKC], vf[2][NDB];
    float scale = 0.f;
    auto load_k = [&](int pa, int pb) __attribute__((always_inline)) {
        const size_t page = (size_t)(lane & 16 ? pb : pa) * page_bytes;
        const u32x4 *p = (const u32x4 *)(k_of + page) + half * 16 + (lane & 15);
#pragma unroll
        for (int x = 0; x < NKC; ++x) kf[x] = p[x * 32];
    };
    auto load_v = [&](int pa, int pb) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const u32x4 *p = (const u32x4 *)(v_of + (size_t)(g ? pb : pa) * page_bytes) + half * 32 + m;
#pragma unroll
            for (int d = 0; d < NDB; ++d) vf[g][d] = p[d * 64];
        }
    };
    auto load_scale = [&](int pa, int pb) __attribute__((always_inline)) {
        scale = *((const float *)((half ? v_of : k_of) + (size_t)(lane & 16 ? pb : pa) * page_bytes + 16 * DH) + (lane & 15));
    };
    if (i0 < i1) {
        fetch_ids(i0);
        const int pa = __builtin_amdgcn_readlane(ida, 0), pb = __builtin_amdgcn_readlane(idb, 0);
        load_scale(pa, pb);
        load_k(pa, pb);
        load_v(pa, pb);
        for (int i = i0; i < i1; ++i) {
            const int base = tiles.at(i) * kStreamTile + 32 * wave;
            const int nx = (i + 1 - i0) & 63;
            if (nx == 0) fetch_ids(i + 1);
            const int na = __builtin_amdgcn_readlane(ida, nx), nb = __builtin_amdgcn_readlane(idb, nx);
            __builtin_amdgcn_wave_barrier();
            scale_of[wave][lane] = scale;
            load_scale(na, nb);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            f32x16 sc[1];
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[0][e] = 0.f;
            int at = lane;
            if (SHARED_Q) asm volatile("" : "+v"(at));   // (read anew for each tile)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                const bf16x8 k = as_bf16(codes8(kf[ks >> 1][2 * (ks & 1)], kf[ks >> 1][2 * (ks & 1) + 1]));
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) sc[0] = mfma32(k, as_bf16(SHARED_Q ? lds.q[ks][t][at] : q[SHARED_Q ? 0 : ks][t]), sc[0]);
            }
            load_k(na, nb);
            if (any_seen<RULES>(r, pre, base)) {
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 x = *(const f32x4 *)&scale_of[wave][2 * e + 4 * half];
#pragma unroll
                    for (int u = 0; u < 4; ++u) sc[0][e + u] *= x[u];
                }
                weigh<RULES, !RULES ? kUnscored : TERMS == 1 ? kScoredRough : kScored, 1, NDT>(a, r, pre, base, sc, run);
                const bool hidden = !all_seen<RULES>(r, pre, base);
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    f32x4 x = *(const f32x4 *)&scale_of[wave][32 + 2 * e + 4 * half];
                    if (hidden) {   // (a scale that is NaN must not meet a weight of 0)
#pragma unroll
                        for (int u = 0; u < 4; ++u) x[u] = sees<RULES>(r, pre, base + 2 * e + 4 * half + u) ? x[u] : 0.f;
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) sc[0][e + u] *= x[u];
                }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = sc[0][8 * g + e];
                    u32x4 w[TERMS];
                    split_terms<TERMS>(x, w);
#pragma unroll
                    for (int d = 0; d < NDT; ++d) {
                        const int odd = 2 * (d & 1);
                        const bf16x8 v = as_bf16(codes8(vf[g][d >> 1][odd], vf[g][d >> 1][odd + 1]));
#pragma unroll
                        for (int t = TERMS - 1; t >= 0; --t) run.o[d] = mfma32(v, as_bf16(w[t]), run.o[d]);
                    }
                }
            }
            load_v(na, nb);
        }
    }
    waves_meet<DH>(a, r, block, kvh, split, tiles.n, run, lds.part, wm, wl);
}

}  // namespace anpd
