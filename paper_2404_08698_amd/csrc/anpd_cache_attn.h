// Attention of new rows over paged caches, and the weight that every cached key receives, for gfx950: the kernels for keys and values in bf16 and fp32.
// What they compute, how rows and products lie in a wave and how exact they are is said in anpd_cache_softmax.h.
#pragma once
#include "anpd_cache_softmax.h"

namespace anpd {

// ------------------------------------------------------------------ few rows: keys and values straight into registers
//
// Block = (32 virtual rows, kv head, split of the keys), four waves; wave w takes keys 32 w .. of every 128.  Nothing is shared
// while the keys go by: a wave's loads are the operands, the next keys are requested when this tile's scores are done, its values
// when its output is, and the waves meet at the end.  This is the form of single tokens, of windows, of prompts whose larger blocks
// would leave compute units without one, and of scores with caps and biases.
// A token or a window is bound by the cache's bytes: 32 tokens of 32 sequences, 271 MB in 51 us (5.4 TB/s), one behind 65535 positions of 8 key heads,
// 268 MB in 49 us (5.5); 17 rows behind 2048, 34 MB in 14 us, are start, three tiles one after the other and end.  A prompt is bound by L2: every
// block reads its keys for 32 rows (512 rows of 32 heads 11 us, 0.19 PFLOP/s).  fp32 rows: three times the matrix instructions; their terms lie in LDS
// once for the four waves, which leaves a wave 192 registers, not 350, and a SIMD two of them: 512 rows 22 -> 15 us, packed documents 49 -> 26.
// grid: n_blocks * n_splits * n_kv_heads
template <int DH, int TERMS, int RULES>
__global__ __launch_bounds__(256, 2) void cache_attn_stream_kernel(const AttnArgs a)
{
    constexpr int NKS = DH / 16, NDT = DH / 32, NDB = DH / 64;
    constexpr bool SHARED_Q = TERMS > 1;   // (the rows' terms in LDS)
    __shared__ union {
        float part[kStreamWaves][2][16][64];   // the waves' outputs, 64 dims at a time
        u32x4 q[SHARED_Q ? NKS : 1][TERMS][64];
    } lds;
    auto &part = lds.part;
    __shared__ float wm[kStreamWaves][32], wl[kStreamWaves][32];
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
    if constexpr (RULES == kTree) tree_info(a, s, pre, parent_of(a, s), depth, r);

    u32x4 q[SHARED_Q ? 1 : NKS][TERMS];
    {
        const size_t at = (size_t)r.row * a.ldq + (size_t)r.head * DH + 8 * half;
        if (SHARED_Q) {
#pragma unroll
            for (int x = 0; x < NKS / kStreamWaves; ++x) {
                const int ks = x * kStreamWaves + wave;
                load_q8<TERMS>(a, at + 16 * ks, q[0]);
#pragma unroll
                for (int t = 0; t < TERMS; ++t) lds.q[ks][t][lane] = q[0][t];
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int ks = 0; ks < (SHARED_Q ? 1 : NKS); ++ks) load_q8<TERMS>(a, at + 16 * ks, q[ks]);
        }
    }
    Running<NDT> run;
    run.start();
    bool unbounded = false;

    const int last_page = (total - 1) >> 4;
    const bf16_t *pool = (const bf16_t *)s.pool;
    const size_t page_elems = (size_t)a.n_layers * 2 * a.n_kv_heads * 16 * DH;
    const bf16_t *k_of = pool + ((size_t)a.layer * 2 * a.n_kv_heads + kvh) * (16 * DH), *v_of = k_of + (size_t)a.n_kv_heads * (16 * DH);
    // physical pages of the wave's next 64 tiles, a tile per lane (beyond the last key: the last page again)
    int ida = 0, idb = 0;
    auto fetch_ids = [&](int i) __attribute__((always_inline)) {
        const int t = i + lane < i1 ? i + lane : i1 - 1;
        const int page = tiles.at(t) * (kStreamTile / 16) + 2 * wave;
        ida = s.table[page < last_page ? page : last_page];
        idb = s.table[page + 1 < last_page ? page + 1 : last_page];
        asm volatile("" : "+v"(ida), "+v"(idb));   // (waited for here: in front of their use all loads in flight would be, at every tile)
    };
    u32x4 kf[NKS], vf[2][NDB][2];   // values: [page][64 dims][keys 4 half.., 8 + 4 half..], two dims side by side
    auto load_k = [&](int pa, int pb) __attribute__((always_inline)) {
        const u32x4 *p = (const u32x4 *)(k_of + (size_t)(lane & 16 ? pb : pa) * page_elems) + half * 16 + (lane & 15);
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) kf[ks] = p[(ks >> 1) * 64 + (ks & 1) * 32];
    };
    auto load_v = [&](int pa, int pb) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const u32x4 *p = (const u32x4 *)(v_of + (size_t)(g ? pb : pa) * page_elems) + (m >> 3) * 32 + half * 8 + (m & 7);
#pragma unroll
            for (int d = 0; d < NDB; ++d)
#pragma unroll
                for (int x = 0; x < 2; ++x) vf[g][d][x] = p[d * 128 + x * 16];
        }
    };
    if (i0 < i1) {
        fetch_ids(i0);
        const int pa = __builtin_amdgcn_readlane(ida, 0), pb = __builtin_amdgcn_readlane(idb, 0);
        load_k(pa, pb);
        load_v(pa, pb);
        for (int i = i0; i < i1; ++i) {
            const int base = tiles.at(i) * kStreamTile + 32 * wave;
            const int nx = (i + 1 - i0) & 63;
            if (nx == 0) fetch_ids(i + 1);
            const int na = __builtin_amdgcn_readlane(ida, nx), nb = __builtin_amdgcn_readlane(idb, nx);
            f32x16 sc[1];
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[0][e] = 0.f;
            int at = lane;
            if (SHARED_Q) asm volatile("" : "+v"(at));   // (read anew for each tile)
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
#pragma unroll
                for (int ks = 0; ks < NKS; ++ks) sc[0] = mfma32(as_bf16(kf[ks]), as_bf16(SHARED_Q ? lds.q[ks][t][at] : q[SHARED_Q ? 0 : ks][t]), sc[0]);
            load_k(na, nb);
            if (any_seen<RULES>(r, pre, base)) {
                weigh<RULES, !RULES ? kUnscored : TERMS == 1 ? kScoredRough : kScored, 1, NDT>(a, r, pre, base, sc, run);
                const bool hidden = !all_seen<RULES>(r, pre, base);
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = sc[0][8 * g + e];
                    u32x4 w[TERMS], v[NDT];
                    split_terms<TERMS>(x, w);
#pragma unroll
                    for (int d = 0; d < NDT; ++d) {
                        const int odd = 2 * (d & 1);
                        v[d] = (u32x4){vf[g][d >> 1][0][odd], vf[g][d >> 1][0][odd + 1], vf[g][d >> 1][1][odd], vf[g][d >> 1][1][odd + 1]};
                    }
                    if (hidden) unbounded |= take_out_unbounded<NDT>(v);
#pragma unroll
                    for (int d = 0; d < NDT; ++d)
#pragma unroll
                        for (int t = TERMS - 1; t >= 0; --t) run.o[d] = mfma32(as_bf16(v[d]), as_bf16(w[t]), run.o[d]);
                }
            }
            load_v(na, nb);
        }
    }
    if (unbounded)
        for (int i = i0; i < i1; ++i) {
            const int base = tiles.at(i) * kStreamTile + 32 * wave;
            if (any_seen<RULES>(r, pre, base) && !all_seen<RULES>(r, pre, base))
                add_unbounded<RULES, NDT>(r, pre, base, run, [&](int d, int e) { return 64 * (d >> 1) + 2 * (8 * (e >> 2) + 4 * half + (e & 3)) + (d & 1); },
                                          [&](int j, int dim) { return bf16_to_f32(v_of[(size_t)s.table[j >> 4] * page_elems + vf_elem(j & 15, dim)]); });
        }
    waves_meet<DH>(a, r, block, kvh, split, tiles.n, run, part, wm, wl);
}

// ------------------------------------------------------------------ many rows: keys and values shared through LDS
//
// Block = (256 bf16 or 128 fp32 virtual rows, kv head, split of the keys), eight or four waves of 32 rows each against the same 32 keys, which go
// from the cache straight into one of eight slots of LDS, six tiles ahead: a key is read from L2 once for the block where the form above
// reads it for 32 rows.  The waves meet at every other tile, where the loads in flight are counted, not waited for.
// 32 keys take a wave about 500 cycles of matrix instructions, as many of vector instructions (a score: a fused product, an exponential,
// a sum, its share of a maximum and of a rounding) and LDS as many for four waves; two waves share a SIMD, which is what the registers
// hold.  One step after the other, the three took turns (each 37 % busy, 143 us for 3584 rows of 32 heads).  So the keys of tile i + 1
// are multiplied while the weights of tile i are formed, and the maximum of tile i + 1 is found while the weights of
// tile i meet its values: both halves of the loop have matrix and vector instructions that do not wait for each other, dealt out in
// turn.  3584 rows of 32 heads now take 117 us, 0.90 PFLOP/s of 105 GFLOP (the library's largest product 1.24); 64 rows per wave, which halves
// what LDS is read for, needed more registers than there are (267 us).
// grid: n_blocks * n_splits * n_kv_heads, blocks with the most keys first
constexpr int kTileKeys = 32;
constexpr int kTileSlots = 8;   // tiles that LDS holds
__host__ __device__ constexpr int tile_waves(int terms) { return terms == 1 ? 8 : 4; }   // what the registers of a SIMD hold
__host__ __device__ constexpr int tile_rows(int terms) { return tile_waves(terms) * kRowTile; }
__host__ __device__ constexpr size_t tile_lds_bytes(int head_dim) { return (size_t)kTileSlots * kTileKeys * head_dim * 4; }

// 16 bytes per lane from p + offset to 1 KB of LDS at byte `at`, past the registers.  In assembly, since behind the builtin the compiler
// lets every read of LDS wait for all loads in flight; what is read is waited for at loads_meet.
__device__ __forceinline__ void load_to_lds(const void *p, uint32_t offset, uint32_t at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(p) : "m0", "memory");
}
// All but the wave's last LEFT loads have arrived, and so have the other waves'; everybody's reads of LDS are done.
template <int LEFT>
__device__ __forceinline__ void loads_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

template <int DH, int TERMS, int RULES>
__global__ __launch_bounds__(tile_waves(TERMS) * 64, tile_waves(TERMS) / 4) void cache_attn_tile_kernel(const AttnArgs a)
{
    constexpr int NKS = DH / 16, NDT = DH / 32, NCH = DH / 32;   // (NCH: 1 KB pieces of a page's keys or values)
    constexpr int WAVES = tile_waves(TERMS), ROWS = WAVES * kRowTile;
    constexpr int LOADS = 4 * NCH / WAVES;   // of a wave for a tile
    extern __shared__ u32x4 lds_tiles[];     // [slot][keys | values][page][piece][lane]
    auto lk = [&](int slot, int page) __attribute__((always_inline)) { return lds_tiles + ((slot * 2 + 0) * 2 + page) * NCH * 64; };
    auto lv = [&](int slot, int page) __attribute__((always_inline)) { return lds_tiles + ((slot * 2 + 1) * 2 + page) * NCH * 64; };
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, m = lane & 31;
    const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int split = rest % a.n_splits, block = a.n_blocks - 1 - rest / a.n_splits;
    const SeqView s = a.seq[seq_of_block(a, block)];
    const int vb = (block - s.block0) * ROWS, rows = s.n * a.group, total = s.pos0 + s.n;
    const int v0 = vb + kRowTile * wave;
    const int p_lo = s.pos0 + vb / a.group, p_hi = s.pos0 + (vb + ROWS <= rows ? vb + ROWS - 1 : rows - 1) / a.group;
    const int pre = RULES && a.prefix > 0 ? (a.prefix < total ? a.prefix : total) : 0;
    const KeyTiles tiles = key_tiles(p_lo, p_hi, total, RULES ? a.window : 0, RULES ? a.prefix : 0, kTileKeys);
    const int begin = split * a.chunk, i1 = begin + a.chunk < tiles.n ? begin + a.chunk : tiles.n;
    if (begin >= tiles.n) return;   // (the whole block; what joins the splits does not look at this one)
    const RowInfo r = row_info<RULES>(a, s, kvh, v0);
    // Tiles f0 .. f1 - 1 are those that every row of the block sees all of.
    int i0 = begin, fk_max = 0;
    if (RULES && TERMS == 1 && a.first_key) {   // (the same for all; with fp32 rows these are the other form's)
        int *lowest = (int *)lds_tiles, *highest = lowest + WAVES;
        const int low = wave_min(r.fk), high = ~wave_min(~r.fk);
        if (lane == 0) { lowest[wave] = low; highest[wave] = high; }
        __syncthreads();
        int fk = lowest[0];
        fk_max = highest[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            fk = lowest[w] < fk ? lowest[w] : fk;
            fk_max = highest[w] > fk_max ? highest[w] : fk_max;
        }
        __syncthreads();
        fk_max = __builtin_amdgcn_readfirstlane(fk_max);
        i0 = first_tile(tiles, __builtin_amdgcn_readfirstlane(fk), begin, i1, kTileKeys);
    }
    int f0, f1;
    {
        const bool window = RULES && a.window > 0;
        const int from = window && p_hi - a.window + 1 > fk_max ? p_hi - a.window + 1 : fk_max, to = window || p_lo >= pre ? p_lo : pre - 1;
        auto place = [&](int t) { return !window ? t : (t <= tiles.b0 ? tiles.a : tiles.a + (t - tiles.b0)); };   // of tile t among those that are visited
        f0 = place(from > 0 ? (from - 1) / kTileKeys + 1 : 0);
        f1 = place((to + 1) / kTileKeys);
        f0 = f0 < i0 ? i0 : f0;
        f0 += (f0 - i0) & 1;   // (tiles are met in twos)
        f0 = f0 < i1 ? f0 : i1;
        f1 = f1 < f0 ? f0 : (f1 < i1 ? f1 : i1);
    }

    u32x4 q[NKS][TERMS];
    {
        const size_t at = (size_t)r.row * a.ldq + (size_t)r.head * DH + 8 * half;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) load_q8<TERMS>(a, at + 16 * ks, q[ks]);
    }
    Running<NDT> run;
    run.start();
    bool unbounded = false;
    const float factor = score_factor<kUnscored>(a);   // (caps and biases are the other form's)

    const int last_page = (total - 1) >> 4;
    const bf16_t *pool = (const bf16_t *)s.pool;
    const size_t page_elems = (size_t)a.n_layers * 2 * a.n_kv_heads * 16 * DH;
    const bf16_t *k_of = pool + ((size_t)a.layer * 2 * a.n_kv_heads + kvh) * (16 * DH), *v_of = k_of + (size_t)a.n_kv_heads * (16 * DH);
    // The wave brings pieces wave, wave + WAVES, ... of a tile: keys of both pages, then values; of one page, or of both in turn.
    // A lane has where that page's keys lie for one of the next 64 tiles from `ids0` on.
    constexpr int PAGES = WAVES < 2 * NCH ? 2 : 1;
    const ptrdiff_t to_values = (ptrdiff_t)a.n_kv_heads * (16 * DH) * sizeof(bf16_t);
    uint32_t at_lo[PAGES], at_hi[PAGES];
    int ids0 = i0;
    auto fetch_ids = [&](int i) __attribute__((always_inline)) {
        const int t = i + lane < i1 ? i + lane : i1 - 1;
#pragma unroll
        for (int x = 0; x < PAGES; ++x) {
            const int page = tiles.at(t) * 2 + (PAGES == 2 ? x : wave / NCH % 2);
            const unsigned long long at = (unsigned long long)(k_of + (size_t)s.table[page < last_page ? page : last_page] * page_elems);
            at_lo[x] = (uint32_t)at;
            at_hi[x] = (uint32_t)(at >> 32);
            asm volatile("" : "+v"(at_lo[x]), "+v"(at_hi[x]));   // (waited for here, not in front of every use)
        }
        ids0 = i;
    };
    const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4 *)lds_tiles) + wave * 1024;
    const uint32_t offset = wave % NCH * 1024 + lane * 16;
    // (beyond the last tile: the last one, for nothing, so that the loads in flight can be counted)
    auto request = [&](int i) __attribute__((always_inline)) {
        const int left = i1 - 1 - ids0, last = left > 0 ? left : 0, x = i - ids0 < last ? i - ids0 : last;   // (addresses fetched behind the last tile: all its own)
        const uint32_t at = lds0 + (uint32_t)((i - i0) & (kTileSlots - 1)) * (4 * NCH * 1024);
#pragma unroll
        for (int c = 0; c < LOADS; ++c) {
            const int y = PAGES == 2 ? c % 2 : 0;
            const char *p = (const char *)(((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)at_hi[y], x) << 32) |
                                           (uint32_t)__builtin_amdgcn_readlane((int)at_lo[y], x));
            // (values: the second half of the pieces, known here but for eight waves of one piece)
            const bool values = LOADS == 1 ? wave >= 2 * NCH : c >= LOADS / 2;
            load_to_lds(values ? p + to_values : p, offset, at + c * WAVES * 1024);
        }
    };
    auto key = [&](int buf, int ks) __attribute__((always_inline)) {
        return as_bf16((lk(buf, (lane >> 4) & 1) + half * 16 + (lane & 15))[(ks >> 1) * 64 + (ks & 1) * 32]);
    };
    auto value = [&](int buf, int g, int d) __attribute__((always_inline)) {
        const uint2 *p = (const uint2 *)lv(buf, g) + (m >> 4) * 64 + half * 16 + (m & 15);
        const uint2 x0 = p[d * 128], x1 = p[d * 128 + 32];
        return (u32x4){x0.x, x0.y, x1.x, x1.y};
    };
    auto products = [&](int buf, f32x16 (&sc)[1]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[0][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            const bf16x8 k = key(buf, ks);
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t) sc[0] = mfma32(k, as_bf16(q[ks][t]), sc[0]);
        }
    };
    // the weights of 32 keys as operands
    auto pack = [&](const f32x16 (&sc)[1], u32x4 (&w)[2][TERMS]) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = sc[0][8 * g + e];
            split_terms<TERMS>(x, w[g]);
        }
    };
    auto any = [&](int i) __attribute__((always_inline)) { return v0 < rows && any_seen<RULES>(r, pre, tiles.at(i) * kTileKeys); };
    auto all = [&](int i) __attribute__((always_inline)) { return all_seen<RULES>(r, pre, tiles.at(i) * kTileKeys); };
    auto slot = [&](int i) __attribute__((always_inline)) { return (i - i0) & (kTileSlots - 1); };
    // Every other tile: tiles i .. i + 2 have arrived, nobody reads those before them any more, and two more are requested (i + 5 was
    // the last one).  Waves that share a SIMD get out of step in between; met at every tile they took turns.
    auto turn = [&](int i) __attribute__((always_inline)) {
        loads_meet<3 * LOADS>();
        if (i + 7 - ids0 >= 64) fetch_ids(i + 6);
        request(i + 6);
        request(i + 7);
    };
    // A tile, one step after the other.
    auto tile = [&](int i) __attribute__((always_inline)) {
        if (((i - i0) & 1) == 0) turn(i);
        if (!any(i)) return;
        f32x16 sc[1];
        u32x4 w[2][TERMS];
        products(slot(i), sc);
        weigh<RULES, kUnscored, 1, NDT>(a, r, pre, tiles.at(i) * kTileKeys, sc, run);
        pack(sc, w);
        const bool hidden = !all(i);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            u32x4 v[NDT];
#pragma unroll
            for (int d = 0; d < NDT; ++d) v[d] = value(slot(i), g, d);
            if (hidden) unbounded |= take_out_unbounded<NDT>(v);
#pragma unroll
            for (int d = 0; d < NDT; ++d)
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) run.o[d] = mfma32(as_bf16(v[d]), as_bf16(w[g][t]), run.o[d]);
        }
    };
    bool huge = false;
    // A tile that all rows see, its products made before, beside the products and the maximum of the next one (`more`).
    auto fused = [&](int i, f32x16 (&sc)[1], f32x16 (&sn)[1], auto more) __attribute__((always_inline)) {
        constexpr bool MORE = decltype(more)::value;
        float f = factor;
        if (huge) {   // (the products rounded here; see huge_reference)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[0][e] *= factor;
            f = 1.f;
        }
        // Written in the order in which it is to run, and held to it: operands from LDS are requested four steps ahead, a step is a
        // matrix instruction (or its terms) and the vector instructions that go beside it.
        constexpr int RING = 4, PV = 2 * NDT, EACH = 16 / NKS;
        const int here = slot(i), there = slot(i + 1);
        __builtin_amdgcn_s_setprio(1);   // (of two waves on a SIMD the one with exponentials to do goes first: 128 -> 124 us)
        u32x4 w[2][TERMS], ring[NKS + PV];
        auto fetch = [&](int x) __attribute__((always_inline)) {
            if (x < NKS) {
                if (MORE) ring[x] = __builtin_bit_cast(u32x4, key(there, x));
            } else if (x < NKS + PV) ring[x] = value(here, (x - NKS) / NDT, (x - NKS) % NDT);
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = MORE ? 0 : NKS; x < (MORE ? 0 : NKS) + RING; ++x) fetch(x);
#pragma unroll
        for (int e = 0; e < 16; ++e) sn[0][e] = 0.f;
        float sum[2] = {0.f, 0.f};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < NKS; ++x) {
            if (MORE) {
                fetch(x + RING);
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) sn[0] = mfma32(as_bf16(ring[x]), as_bf16(q[x][t]), sn[0]);
            }
#pragma unroll
            for (int e = EACH * x; e < EACH * (x + 1); e += 2) {
                const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[0][e], f, -run.m)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[0][e + 1], f, -run.m));
                sum[0] += p0;
                sum[1] += p1;
                uint32_t t[TERMS];
                split_pair<TERMS>(p0, p1, t);
#pragma unroll
                for (int k = 0; k < TERMS; ++k) w[e >> 3][k][(e & 7) >> 1] = t[k];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        run.l += sum[0] + sum[1];
        __builtin_amdgcn_s_setprio(0);
        float mx = -INFINITY;
#pragma unroll
        for (int y = 0; y < PV; ++y) {
            fetch(NKS + y + RING);
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t) run.o[y % NDT] = mfma32(as_bf16(ring[NKS + y]), as_bf16(w[y / NDT][t]), run.o[y % NDT]);
            if (MORE) {   // (the products need a step or two before they are there)
                constexpr int LATE = PV / 4;
#pragma unroll
                for (int e = y < LATE ? 0 : 16 * (y - LATE) / (PV - LATE); e < (y < LATE ? 0 : 16 * (y - LATE + 1) / (PV - LATE)); ++e) mx = fmaxf(mx, sn[0][e]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (MORE) {
            mx = both_halves_max(mx) * factor;
            if (__builtin_amdgcn_ballot_w64(mx > run.m + 8.f) != 0) {
                move_reference(run, mx > run.m + 8.f ? mx : run.m);
                huge = huge_reference(run.m);
            }
        }
    };
    if (i0 < i1) {
        fetch_ids(i0);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 6; ++t) request(i0 + t);
        for (int i = i0; i < f0; ++i) tile(i);
        if (f0 < f1) {
            f32x16 s0[1], s1[1];
            if (f0 == i0) loads_meet<5 * LOADS>();   // (later tiles have arrived with the turn before)
            products(slot(f0), s0);
            move_reference(run, new_reference<1>(s0, factor, run.m));
            huge = huge_reference(run.m);
            int i = f0;
            for (; i + 2 < f1; i += 2) {
                turn(i);
                fused(i, s0, s1, std::true_type());
                fused(i + 1, s1, s0, std::true_type());
            }
            turn(i);
            if (i + 1 < f1) {
                fused(i, s0, s1, std::true_type());
                fused(i + 1, s1, s0, std::false_type());
            } else fused(i, s0, s1, std::false_type());
        }
        for (int i = f1; i < i1; ++i) tile(i);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (LDS must not be given up while something is on its way to it)
    if (unbounded)
        for (int i = i0; i < i1; ++i)
            if (any(i) && !all(i))
                add_unbounded<RULES, NDT>(r, pre, tiles.at(i) * kTileKeys, run, [&](int d, int e) { return 32 * d + 8 * (e >> 2) + 4 * half + (e & 3); },
                                          [&](int j, int dim) { return bf16_to_f32(v_of[(size_t)s.table[j >> 4] * page_elems + vf_elem(j & 15, dim)]); });
    const float l = both_halves_sum(run.l);
    if (!r.live) return;
    if (a.part && tiles.n > a.chunk) {   // (otherwise this split is all there is)
        float *to = a.part + (((size_t)block * a.n_kv_heads + kvh) * a.n_splits + split) * part_floats(ROWS, DH);
        const int row = kRowTile * wave + m;
        if (half == 0) *(float2 *)(to + ROWS * DH + 2 * row) = make_float2(run.m, l);
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(f32x4 *)(to + row * DH + 32 * d + 8 * i + 4 * half) = (f32x4){run.o[d][4 * i], run.o[d][4 * i + 1], run.o[d][4 * i + 2], run.o[d][4 * i + 3]};
    } else {
        const float inv = inverse_sum(l);
        if (half == 0) store_lse(a, r.row, r.head, run.m, l);
#pragma unroll
        for (int d = 0; d < NDT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                store_out4(a, DH, r.row, r.head, 32 * d + 8 * i + 4 * half, (f32x4){run.o[d][4 * i], run.o[d][4 * i + 1], run.o[d][4 * i + 2], run.o[d][4 * i + 3]} * inv);
    }
}

// ------------------------------------------------------------------ caches in plain order
//
// Blocks of [token][dim] in fp32 or bf16, pages of 8 to 256 tokens: exact fp32 products (v_mfma_f32_32x32x2_f32, whose lanes hold
// the same rows and keys as above).  The two contracted numbers of an instruction are dims t and t + head_dim / 2 of a key, so a lane
// reads half a key in one piece.  Blocks, waves and splits as in the form for few rows, whatever the rows' number.
// grid: n_blocks * n_splits * n_kv_heads
__device__ __forceinline__ f32x16 mfma32f(float x, float y, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(x, y, c, 0, 0, 0); }

template <int DH>
__device__ __forceinline__ void load_half(const float *p, float (&x)[DH / 2])
{
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) {
        const f32x4 u = ((const f32x4 *)p)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] = u[e];
    }
}
template <int DH>
__device__ __forceinline__ void load_half(const bf16_t *p, float (&x)[DH / 2])
{
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) {
        const u32x4 u = ((const u32x4 *)p)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[8 * i + 2 * e] = __uint_as_float(u[e] << 16); x[8 * i + 2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u); }
    }
}

template <typename KT, int DH, int RULES>
__global__ __launch_bounds__(256, 1) void cache_attn_plain_kernel(const AttnArgs a)
{
    constexpr int NDT = DH / 32;
    __shared__ float part[kStreamWaves][16][64];
    __shared__ float wm[kStreamWaves][32], wl[kStreamWaves][32];
    __shared__ int depth[RULES == kTree ? kTreeRows : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, m = lane & 31;
    const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int split = rest % a.n_splits, block = a.n_blocks - 1 - rest / a.n_splits;
    const SeqView s = a.seq[seq_of_block(a, block)];
    const int v0 = (block - s.block0) * kRowTile, total = s.pos0 + s.n, pt = a.page_tokens;
    RowInfo r = row_info<RULES>(a, s, kvh, v0);
    const int pre = a.prefix > 0 ? (a.prefix < total ? a.prefix : total) : 0;
    const KeyTiles tiles = key_tiles(a, s, __builtin_amdgcn_readlane(r.p, 0), __builtin_amdgcn_readlane(r.p, 31), kStreamTile);
    const int begin = split * a.chunk, i1 = begin + a.chunk < tiles.n ? begin + a.chunk : tiles.n;
    if (begin >= tiles.n) return;
    const int i0 = first_tile(tiles, wave_min(r.fk), begin, i1, kStreamTile);
    if constexpr (RULES == kTree) tree_info(a, s, pre, parent_of(a, s), depth, r);
    float q[DH / 2];
    {
        const size_t at = (size_t)r.row * a.ldq + (size_t)r.head * DH + half * (DH / 2);
#pragma unroll
        for (int i = 0; i < DH / 16; ++i) {
            float x[8];
            load_q8(a, at + 8 * i, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) q[8 * i + e] = x[e];
        }
    }
    Running<NDT> run;
    run.start();
    bool unbounded = false;
    const KT *pool = (const KT *)s.pool;
    for (int i = i0; i < i1; ++i) {
        const int base = tiles.at(i) * kStreamTile + 32 * wave;
        if (!any_seen<RULES>(r, pre, base)) continue;
        // (all of the tile's loads before the first product: one at a time, between the products, they were most of the time)
        float v[16][NDT];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = base + 8 * (e >> 2) + 4 * half + (e & 3), key = j < total ? j : total - 1;
            const KT *p = pool + kv_offset(s.table[key / pt], a.layer, a.n_layers, 1, kvh, a.n_kv_heads, key % pt, pt, DH) + m;
#pragma unroll
            for (int d = 0; d < NDT; ++d) v[e][d] = load_f32(p, 32 * d);
        }
        f32x16 sc[1];
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[0][e] = 0.f;
        {
            const int key = base + m < total ? base + m : total - 1;
            float k[DH / 2];
            load_half<DH>(pool + kv_offset(s.table[key / pt], a.layer, a.n_layers, 0, kvh, a.n_kv_heads, key % pt, pt, DH) + half * (DH / 2), k);
#pragma unroll
            for (int t = 0; t < DH / 2; ++t) sc[0] = mfma32f(k[t], q[t], sc[0]);
        }
        weigh<RULES, kScored, 1, NDT>(a, r, pre, base, sc, run);
        if (!all_seen<RULES>(r, pre, base))
#pragma unroll
            for (int e = 0; e < 16; ++e)
#pragma unroll
                for (int d = 0; d < NDT; ++d) {
                    const bool fin = fabsf(v[e][d]) <= 3.4028234e38f;
                    unbounded |= __builtin_amdgcn_ballot_w64(!fin) != 0;
                    v[e][d] = fin ? v[e][d] : 0.f;
                }
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int d = 0; d < NDT; ++d) run.o[d] = mfma32f(v[e][d], sc[0][e], run.o[d]);
    }
    if (unbounded)
        for (int i = i0; i < i1; ++i) {
            const int base = tiles.at(i) * kStreamTile + 32 * wave;
            if (any_seen<RULES>(r, pre, base) && !all_seen<RULES>(r, pre, base))
                add_unbounded<RULES, NDT>(r, pre, base, run, [&](int d, int e) { return 32 * d + 8 * (e >> 2) + 4 * half + (e & 3); }, [&](int j, int dim) {
                    return load_f32(pool + kv_offset(s.table[j / pt], a.layer, a.n_layers, 1, kvh, a.n_kv_heads, j % pt, pt, DH), dim);
                });
        }
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
    float *to = a.part && tiles.n > a.chunk ? a.part + (((size_t)block * a.n_kv_heads + kvh) * a.n_splits + split) * part_floats(kRowTile, DH) : nullptr;
    if (wave == 0 && half == 0 && r.live) {   // (beyond the last row nobody asks)
        if (to) *(float2 *)(to + kRowTile * DH + 2 * m) = make_float2(top, sum);
        else store_lse(a, r.row, r.head, top, sum);
    }
    const float inv = inverse_sum(sum);
#pragma unroll
    for (int d = 0; d < NDT; ++d) {
        if (d > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) part[wave][i][lane] = run.o[d][i] * f;
        __syncthreads();
        f32x4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = part[0][4 * wave + i][lane];
#pragma unroll
            for (int w = 1; w < kStreamWaves; ++w) x[i] += part[w][4 * wave + i][lane];
        }
        const int dim = 32 * d + 8 * wave + 4 * half;
        if (!r.live) continue;
        if (to) *(f32x4 *)(to + m * DH + dim) = x;
        else store_out4(a, DH, r.row, r.head, dim, x * inv);
    }
}

// ------------------------------------------------------------------ the splits meet
//
// Four adjacent dims of a row per thread.  TOGETHER: a block per row, the splits dealt to its groups of DH / 4 threads, whose sums
// meet in LDS in their order, for few rows of many splits (with a block for all rows of a key / value head and the splits one after the
// other a token behind 65535 positions waited 23 us for 128 of them, so 5).  Otherwise a group has a row to itself: 1536 rows of 32 heads
// in two or three splits took 70 us with a block for each row.
// row_block: rows of the blocks that were split; tile: keys of their tiles.
// grid: n_kv_heads * n_blocks * (row_block, or row_block / rows of a block)
template <int DH, bool TOGETHER>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(const AttnArgs a, int row_block, int tile)
{
    constexpr int TPR = DH / 4, GROUPS = 256 / TPR, STEP = TOGETHER ? GROUPS : 1;
    __shared__ float tops[GROUPS], sums[GROUPS];
    __shared__ f32x4 part[GROUPS][TPR];
    const int group = threadIdx.x / TPR, d = threadIdx.x % TPR;
    const int per = TOGETHER ? row_block : row_block / GROUPS;
    const int row = TOGETHER ? blockIdx.x % per : blockIdx.x % per * GROUPS + group, rest = blockIdx.x / per, kvh = rest % a.n_kv_heads, block = rest / a.n_kv_heads;
    const SeqView s = a.seq[seq_of_block(a, block)];
    const int vb = (block - s.block0) * row_block, rows = s.n * a.group, v = vb + row;
    if (v >= rows) return;   // (TOGETHER: the whole block)
    const int p_lo = s.pos0 + vb / a.group, p_hi = s.pos0 + (vb + row_block <= rows ? vb + row_block - 1 : rows - 1) / a.group;
    const KeyTiles tiles = key_tiles(a, s, p_lo, p_hi, tile);
    const int used = (tiles.n + a.chunk - 1) / a.chunk;
    if (used < 2) return;   // (written by the split itself)
    const size_t stride = part_floats(row_block, DH);
    const float *from = a.part + ((size_t)block * a.n_kv_heads + kvh) * a.n_splits * stride;
    const float *ml = from + row_block * DH + 2 * row, *o = from + row * DH + 4 * d;
    float top = kNoKey, sum = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    // (requested side by side, four splits at a time; one that does not exist weighs nothing)
    for (int k0 = TOGETHER ? group : 0; k0 < used; k0 += 4 * STEP) {
        float2 t[4];
        f32x4 y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int k = k0 + u * STEP < used ? k0 + u * STEP : k0;
            t[u] = *(const float2 *)(ml + k * stride);
            y[u] = *(const f32x4 *)(o + k * stride);
        }
        float t0 = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) t0 = fmaxf(t0, t[u].x);
        const float f0 = __builtin_amdgcn_exp2f(top - t0);
        top = t0;
        sum *= f0;
        x = x * f0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (k0 + u * STEP >= used) continue;
            const float f = __builtin_amdgcn_exp2f(t[u].x - t0);
            sum = fmaf(t[u].y, f, sum);
            x += y[u] * f;
        }
    }
    if constexpr (TOGETHER) {
        if (d == 0) { tops[group] = top; sums[group] = sum; }
        part[group][d] = x;
        __syncthreads();
        if (group > 0) return;
        top = tops[0];
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) top = fmaxf(top, tops[g]);
        sum = 0.f;
        x = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const float f = __builtin_amdgcn_exp2f(tops[g] - top);
            sum = fmaf(sums[g], f, sum);
            x += part[g][d] * f;
        }
    }
    const int r = v / a.group, out_row = s.row0 + r, head = kvh * a.group + (v - r * a.group);
    if (d == 0) store_lse(a, out_row, head, top, sum);
    store_out4(a, DH, out_row, head, 4 * d, x * inverse_sum(sum));
}

// ------------------------------------------------------------------ the weight of every key
//
// Block = (128 SETS keys, kv head, part of the rows), four waves of SETS x 32 keys, whose operands a wave holds in registers while the
// rows go by in tiles of 32 through LDS (fp32 rows are split into their terms there, once for the four waves).  A lane adds the weights
// of its row's 16 keys per set to as many sums over all tiles; the lanes meet at the end.  Two sets use a row operand twice for
// one read of it: with one, LDS was as busy as the matrix cores (1800 fp32 rows of 40 heads 127 us, with two 75: 50 GFLOP of terms at
// 0.66 PFLOP/s).  One block owns a key's sum, so there are no atomics and the order is always the same; where keys are too few for all compute units, the rows are dealt to several blocks whose sums are
// added in order by a second kernel.  exp(t - lse) is formed from the difference, not from two numbers scaled to base 2 first,
// whose roundings would stay in it.
// a.block0 / n_blocks / n_splits / chunk: blocks of keys; parts of the rows, row tiles in each.
// grid: n_blocks * n_splits * n_kv_heads
constexpr int kMassKeys = 128;   // of a block, per set

// The row tiles that can see keys kb .. kb + keys - 1: first one and one behind the last.
struct RowTiles {
    int t0, t1;
};
__host__ __device__ __forceinline__ RowTiles row_tiles(int kb, int keys, int pos0, int n, int group, int window, int prefix)
{
    const long long rows = (long long)n * group;
    long long v0 = 0, v1 = rows;
    if (kb >= prefix) {
        v0 = (long long)(kb - pos0) * group;
        if (v0 < 0) v0 = 0;
        if (window > 0) {
            v1 = ((long long)kb + keys - 1 + window - pos0) * group;
            if (v1 > rows) v1 = rows;
        }
    }
    RowTiles t;
    t.t0 = (int)(v0 / kRowTile);
    t.t1 = v1 > v0 ? (int)((v1 + kRowTile - 1) / kRowTile) : t.t0;
    return t;
}

// The lane's row in a sum of weights.  No row, or one whose lse says that it adds nothing, sees no key: an infinite or NaN product of what
// it holds would not become 0 by any lse.  (A selection in add_weights on its own: 1800 fp32 rows of 40 heads 74 -> 78 us.)
__device__ __forceinline__ RowInfo row_in_sum(RowInfo r, float lse)
{
    if (!r.live || fabsf(lse) == INFINITY) {
        r.p = -1;
        r.fk = r.lo = 0x7fffffff;
    }
    return r;
}

// Weights of the lane's 16 keys, added to `acc`.
template <bool RULES>
__device__ __forceinline__ void add_weights(const AttnArgs &a, const RowInfo &r, float lse, int pre, int base, const f32x16 &s, f32x16 &acc)
{
    const int half = (threadIdx.x >> 5) & 1;
    const bool scored = RULES && (a.cap > 0.f || a.slopes);
    if (!scored && all_seen<RULES>(r, pre, base)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] += __builtin_amdgcn_exp2f(fmaf(s[i], a.scale, -lse) * kLog2e);
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int j = base + 8 * (i >> 2) + 4 * half + (i & 3);
        const float t = scored ? ruled_score<false>(a, s[i], r.slope, r.p - j) - lse : fmaf(s[i], a.scale, -lse);
        acc[i] += sees<RULES>(r, pre, j) ? __builtin_amdgcn_exp2f(t * kLog2e) : 0.f;
    }
}

// The lanes' sums meet: key k of the wave's 32 for lanes 0 .. 31; `red`: the wave's own kilobytes.
__device__ __forceinline__ float meet_lanes(const f32x16 &acc, float (&red)[16][64])
{
    const int lane = threadIdx.x & 63, k = lane & 31, from = (k >> 3) * 4 + (k & 3), half = (k >> 2) & 1;
#pragma unroll
    for (int i = 0; i < 16; ++i) red[i][lane] = acc[i];
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < 32; ++x) sum += red[from][half * 32 + ((x + k) & 31)];   // (turned by k: every lane its own bank)
    return sum;
}
// k: key of the block, key: of the sequence
__device__ __forceinline__ void store_mass(const AttnArgs &a, const MassOut &to, int seq, int total, int kvh, int block, int split, int keys, int k, int key, float sum)
{
    if (a.part) a.part[(((size_t)block * a.n_kv_heads + kvh) * a.n_splits + split) * keys + k] = sum;
    else if (key < total) to.mass[seq][(size_t)kvh * to.ld + key] += sum;
}

template <int DH, int TERMS, bool RULES, int SETS>
__global__ __launch_bounds__(256, 2) void cache_mass_kernel(const AttnArgs a, const MassOut to)
{
    constexpr int NKS = DH / 16, UNITS = NKS * 64 / 256;   // pieces of eight dims of a row tile per thread
    __shared__ union {
        u32x4 q[2][TERMS][NKS][64];
        float red[4][16][64];
    } lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, m = lane & 31;
    const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int split = rest % a.n_splits, block = rest / a.n_splits, seq = seq_of_block(a, block);
    const SeqView s = a.seq[seq];
    const int kb = (block - s.block0) * (kMassKeys * SETS), base = kb + 32 * SETS * wave, total = s.pos0 + s.n;
    const int pre = RULES && a.prefix > 0 ? (a.prefix < total ? a.prefix : total) : 0;
    const RowTiles tiles = row_tiles(kb, kMassKeys * SETS, s.pos0, s.n, a.group, RULES ? a.window : 0, pre);
    const int t0 = tiles.t0 + split * a.chunk, t1 = t0 + a.chunk < tiles.t1 ? t0 + a.chunk : tiles.t1;
    if (t0 >= tiles.t1) return;   // (the whole block)

    u32x4 kf[SETS][NKS];
#pragma unroll
    for (int x = 0; x < SETS; ++x) {
        const int last_page = (total - 1) >> 4, page = ((base + 32 * x) >> 4) + ((lane >> 4) & 1);
        const int id = s.table[page < last_page ? page : last_page];
        const bf16_t *pool = (const bf16_t *)s.pool + kvf_base(id, a.layer, a.n_layers, 0, kvh, a.n_kv_heads, DH);
        const u32x4 *p = (const u32x4 *)pool + half * 16 + (lane & 15);
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) kf[x][ks] = p[(ks >> 1) * 64 + (ks & 1) * 32];
    }
    // what the next tile is made of, as it comes from memory (nothing is done to it before the tile at hand is through): its rows' pieces,
    // and every lane's row
    u32x4 piece[UNITS][1];
    float wide[UNITS][8];
    RowInfo r_next;
    float lse_next = 0.f;
    auto request = [&](int t) __attribute__((always_inline)) {
        r_next = row_info<RULES>(a, s, kvh, t * kRowTile);
        const size_t at = (size_t)r_next.row * a.ldq + (size_t)r_next.head * DH + 8 * half;
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if constexpr (TERMS == 1) load_q8<1>(a, at + 16 * (wave + 4 * u), piece[u]);
            else load_q8(a, at + 16 * (wave + 4 * u), wide[u]);
        }
        lse_next = a.lse[(size_t)r_next.row * a.n_heads + r_next.head];
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            u32x4 t[TERMS];
            if constexpr (TERMS == 1) t[0] = piece[u][0];
            else split_terms<TERMS>(wide[u], t);
#pragma unroll
            for (int k = 0; k < TERMS; ++k) lds.q[buf][k][wave + 4 * u][lane] = t[k];
        }
    };
    f32x16 acc[SETS] = {};
    request(t0);
    put(0);
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        const float lse = lse_next;
        const RowInfo r = row_in_sum(r_next, lse);
        __syncthreads();
        if (t + 1 < t1) request(t + 1);
        bool seen = false;
#pragma unroll
        for (int x = 0; x < SETS; ++x) seen = seen || (base + 32 * x < total && any_seen<RULES>(r, pre, base + 32 * x));
        if (seen) {
            f32x16 sc[SETS] = {};
#pragma unroll
            for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                for (int ks = 0; ks < NKS; ++ks) {
                    const bf16x8 q = as_bf16(lds.q[buf][k][ks][lane]);
#pragma unroll
                    for (int x = 0; x < SETS; ++x) sc[x] = mfma32(as_bf16(kf[x][ks]), q, sc[x]);
                }
#pragma unroll
            for (int x = 0; x < SETS; ++x) add_weights<RULES>(a, r, lse, pre, base + 32 * x, sc[x], acc[x]);
        }
        if (t + 1 < t1) put(buf ^ 1);
    }
#pragma unroll
    for (int x = 0; x < SETS; ++x) {
        __syncthreads();
        const float sum = meet_lanes(acc[x], lds.red[wave]);
        const int k = 32 * (SETS * wave + x) + m;
        if (half == 0) store_mass(a, to, seq, total, kvh, block, split, kMassKeys * SETS, k, kb + k, sum);
    }
}

// The same for caches in plain order (exact fp32 products).
template <typename KT, int DH>
__global__ __launch_bounds__(256, 1) void cache_mass_plain_kernel(const AttnArgs a, const MassOut to)
{
    constexpr int N8 = DH / 16, UNITS = N8 * 64 / 256;
    __shared__ union {
        f32x4 q[2][DH / 8][64];   // [four of the lane's half row][lane]
        float red[4][16][64];
    } lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, m = lane & 31;
    const int kvh = blockIdx.x % a.n_kv_heads, rest = blockIdx.x / a.n_kv_heads;
    const int split = rest % a.n_splits, block = rest / a.n_splits, seq = seq_of_block(a, block);
    const SeqView s = a.seq[seq];
    const int kb = (block - s.block0) * kMassKeys, base = kb + 32 * wave, total = s.pos0 + s.n, pt = a.page_tokens;
    const int pre = a.prefix > 0 ? (a.prefix < total ? a.prefix : total) : 0;
    const RowTiles tiles = row_tiles(kb, kMassKeys, s.pos0, s.n, a.group, a.window, pre);
    const int t0 = tiles.t0 + split * a.chunk, t1 = t0 + a.chunk < tiles.t1 ? t0 + a.chunk : tiles.t1;
    if (t0 >= tiles.t1) return;   // (the whole block)
    float k[DH / 2];
    {
        const int key = base + m < total ? base + m : total - 1;
        load_half<DH>((const KT *)s.pool + kv_offset(s.table[key / pt], a.layer, a.n_layers, 0, kvh, a.n_kv_heads, key % pt, pt, DH) + half * (DH / 2), k);
    }
    float piece[UNITS][8];
    RowInfo r_next;
    float lse_next = 0.f;
    auto request = [&](int t) __attribute__((always_inline)) {
        r_next = row_info<true>(a, s, kvh, t * kRowTile);
        const size_t at = (size_t)r_next.row * a.ldq + (size_t)r_next.head * DH + half * (DH / 2);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) load_q8(a, at + 8 * (wave + 4 * u), piece[u]);
        lse_next = a.lse[(size_t)r_next.row * a.n_heads + r_next.head];
    };
    auto put = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                lds.q[buf][2 * (wave + 4 * u) + e][lane] = (f32x4){piece[u][4 * e], piece[u][4 * e + 1], piece[u][4 * e + 2], piece[u][4 * e + 3]};
    };
    f32x16 acc = {};
    request(t0);
    put(0);
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        const float lse = lse_next;
        const RowInfo r = row_in_sum(r_next, lse);
        __syncthreads();
        if (t + 1 < t1) request(t + 1);
        if (base < total && any_seen<true>(r, pre, base)) {
            f32x16 sc = {};
#pragma unroll
            for (int i = 0; i < DH / 8; ++i) {
                const f32x4 q = lds.q[buf][i][lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) sc = mfma32f(k[4 * i + e], q[e], sc);
            }
            add_weights<true>(a, r, lse, pre, base, sc, acc);
        }
        if (t + 1 < t1) put(buf ^ 1);
    }
    __syncthreads();
    const float sum = meet_lanes(acc, lds.red[wave]);
    if (half == 0) store_mass(a, to, seq, total, kvh, block, split, kMassKeys, 32 * wave + m, base + m, sum);
}

// The parts of the rows meet, in their order.   grid: n_blocks * n_kv_heads, a thread per key of the block
__global__ void cache_mass_join_kernel(const AttnArgs a, const MassOut to)
{
    const int kvh = blockIdx.x % a.n_kv_heads, block = blockIdx.x / a.n_kv_heads, seq = seq_of_block(a, block), keys = blockDim.x;
    const SeqView s = a.seq[seq];
    const int kb = (block - s.block0) * keys, total = s.pos0 + s.n, key = kb + (int)threadIdx.x;
    const int pre = a.prefix < total ? a.prefix : total;
    const RowTiles tiles = row_tiles(kb, keys, s.pos0, s.n, a.group, a.window, pre);
    const int used = (tiles.t1 - tiles.t0 + a.chunk - 1) / a.chunk;
    const float *from = a.part + ((size_t)block * a.n_kv_heads + kvh) * a.n_splits * keys + threadIdx.x;
    float sum = 0.f;
#pragma unroll 4
    for (int k = 0; k < used; ++k) sum += from[(size_t)k * keys];
    if (key < total && used > 0) to.mass[seq][(size_t)kvh * to.ld + key] += sum;
}

// ------------------------------------------------------------------ rows of a prompt
//
// The last rows of a prompt out of its queries' split operand [head][row group][dims / 32][hi | lo][lane][8] (lane = 16 * (dims % 32 / 8) +
// row of the group) as fp32 rows [n][heads * DH]; m0: first one among the operand's rows.   grid: (n, heads), DH threads
__global__ void prompt_rows_kernel(const bf16_t *__restrict__ qp, float *__restrict__ q, int G, int m0, int head_dim)
{
    const int r = blockIdx.x, head = blockIdx.y, dim = threadIdx.x, m = m0 + r;
    const size_t at = ((((size_t)head * G + (m >> 4)) * (head_dim >> 5) + (dim >> 5)) * 2 * 64 + ((dim >> 3) & 3) * 16 + (m & 15)) * 8 + (dim & 7);
    q[((size_t)r * gridDim.y + head) * head_dim + dim] = bf16_to_f32(qp[at]) + bf16_to_f32(qp[at + 64 * 8]);
}

}  // namespace anpd
