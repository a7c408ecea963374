// Eviction from a cache: which positions stay, and their keys and values moved together, for gfx950.
//
// Per layer and key / value head the first `first` positions, the last `last` and, of those between, the ones with the largest mass
// stay (equal ones: the lowest position), in their order: the positions of a head's slots differ from head to head.
// A key that moves from position p to slot i can be turned by the difference, k' = R((i - p) theta) k, theta_n = base^(-2 n / dim), so
// that it is the key of a token at position i.
#pragma once
#include "anpd_layout.h"

namespace anpd {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// Numbers as integers of the same order; NaN below all of them, -0 is 0.
__device__ __forceinline__ uint32_t mass_rank(float x)
{
    if (x != x) return 0;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float mass_of_rank(uint32_t r) { return r == 0 ? __builtin_nanf("") : __uint_as_float(r & 0x80000000u ? r & 0x7fffffffu : ~r); }

// n and the lanes of the mask before this one
__device__ __forceinline__ uint32_t lanes_below(unsigned long long mask, uint32_t n)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, n));
}

struct SelectArgs {
    const float *mass;   // [layer][head][ld]
    int32_t *kept;       // [layer][head][keep]
    float *out_mass;     // [layer][head][ld_out] or NULL
    int64_t ld, ld_out;
    int32_t len, keep, first, last;
};

// Block = (layer, head); a wave has a stretch of whole 64s of positions.  What stays in any case has the highest rank of all, so that
// one search finds the smallest rank that stays; then every wave counts what stays of its stretch, the counts are summed over the
// waves, and each wave writes its own.
// HELD: positions per lane, whose ranks stay in registers: the search goes bit by bit, a comparison and a count of the lanes per 64 positions,
// and ends as soon as a rank separates as many as are wanted.  HELD = 0 (beyond 65536 positions): byte by byte, each time with a
// histogram of the candidates' next byte in LDS (whole numbers: the order of the counts does not matter), for which all is
// read again.  8 heads of 65536 positions: 132 us with the histogram, 64 with registers, of them 9 to load, 30 for some 22 steps of the search
// (64 comparisons a wave, and a meeting of the waves), 18 to write; 64 heads of 3584 14 us, a step 0.4 of them, the meeting.
// grid: n_layers * n_kv_heads
template <int HELD>
__global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(const SelectArgs a)
{
    __shared__ uint32_t bins[256], above[kSelectWaves], equal[kSelectWaves], choice[2];
    __shared__ uint4 counts[2][kSelectWaves / 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *mass = a.mass + (size_t)blockIdx.x * a.ld;
    int32_t *kept = a.kept + (size_t)blockIdx.x * a.keep;
    float *out = a.out_mass ? a.out_mass + (size_t)blockIdx.x * a.ld_out : nullptr;
    const uint32_t want = (uint32_t)a.keep;
    const int steps = (a.len + kSelectThreads - 1) / kSelectThreads, p0 = wave * steps * 64;   // positions p0 + 64 k + lane, k < steps
    // (a position behind the last one has the lowest rank and comes last among those: it never stays)
    const int p1 = p0 + 64 * steps < a.len ? p0 + 64 * steps : a.len;
    auto load = [&](int k) __attribute__((always_inline)) {
        const int i = p0 + 64 * k + lane;
        return mass[i < a.len ? i : a.len - 1];
    };
    auto rank_of = [&](int k, float x) __attribute__((always_inline)) {
        const int i = p0 + 64 * k + lane;
        return i >= p1 ? 0u : (i < a.first || i >= a.len - a.last ? ~0u : mass_rank(x));
    };
    uint32_t held[HELD > 0 ? HELD : 1];
#pragma unroll
    for (int k = 0; k < HELD; ++k) held[k] = __float_as_uint(load(k));
#pragma unroll
    for (int k = 0; k < HELD; ++k) {
        held[k] = rank_of(k, __uint_as_float(held[k]));
        __builtin_amdgcn_sched_barrier(0);
    }
    // fn(position, rank) for the wave's stretch, 64 positions at a time
    auto each = [&](auto fn) __attribute__((always_inline)) {
        if constexpr (HELD > 0) {
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                if (k < steps) fn(p0 + 64 * k + lane, held[k]);   // (the same for the whole wave)
                __builtin_amdgcn_sched_barrier(0);   // (one after the other: the ranks fill the registers)
            }
        } else {
            for (int k0 = 0; k0 < steps; k0 += 8) {
                uint32_t y[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) y[u] = __float_as_uint(load(k0 + u));
#pragma unroll
                for (int u = 0; u < 8; ++u) y[u] = rank_of(k0 + u, __uint_as_float(y[u]));
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (k0 + u < steps) fn(p0 + 64 * (k0 + u) + lane, y[u]);
            }
        }
    };
    uint32_t limit = 0, left = want;   // ranks above `limit` stay, and `left` of those equal to it
    if constexpr (HELD > 0) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t t = limit | (1u << bit);
            // (two of three are counted by the scalar unit, which the compute unit's waves share, the third by the lanes themselves)
            uint32_t n = 0, own = 0;
#pragma unroll
            for (int k = 0; k < HELD; ++k) {
                if (HELD >= 16 && k % 3 == 2) {
                    own += held[k] >= t ? 1u : 0u;
                    asm volatile("" : "+s"(n), "+v"(own));   // (all comparisons first would be more than the scalar registers hold)
                } else n += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(held[k] >= t));
            }
            if (HELD >= 16) {
#pragma unroll
                for (int b = 0; b < 5; ++b) n += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64((own >> b) & 1u)) << b;   // (21 at most)
            }
            if (lane == 0) ((uint32_t *)counts[bit & 1])[wave] = n;
            __syncthreads();   // (the other half of the counts is read until the next one)
            uint32_t total = 0;
#pragma unroll
            for (int w = 0; w < kSelectWaves / 4; ++w) { const uint4 c = counts[bit & 1][w]; total += (c.x + c.y) + (c.z + c.w); }
            total = (uint32_t)__builtin_amdgcn_readfirstlane((int)total);
            if (total == want) {   // (the same for all)
                limit = t - 1;
                left = 0;
                break;
            }
            if (total > want) limit = t;
            else left = want - total;   // (of the ranks above the limit that is found in the end, this many are missing)
        }
    } else {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) bins[tid] = 0;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
            each([&](int i, uint32_t rank) __attribute__((always_inline)) {
                const bool in = (rank & mask) == limit && i < a.len;
                const uint32_t bin = (rank >> shift) & 255u;
                // (the first candidate's bin at once for all lanes that share it: positions that nothing looked at are all 0)
                const unsigned long long some = __builtin_amdgcn_ballot_w64(in);
                if (some == 0) return;
                const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)bin, __builtin_ctzll(some));
                const unsigned long long same = __builtin_amdgcn_ballot_w64(in && bin == one);
                if (lane == 0) atomicAdd(&bins[one], (uint32_t)__builtin_popcountll(same));
                if (in && bin != one) atomicAdd(&bins[bin], 1u);
            });
            __syncthreads();
            if (wave == 0) {
                // from the top bin down: the one in which the `left`th candidate lies.  Lane: four bins, the highest first.
                uint32_t n[4], sum = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) { n[k] = bins[255 - 4 * lane - k]; sum += n[k]; }
                uint32_t before = sum;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) { const uint32_t t = (uint32_t)__shfl_up((int)before, o, 64); if (lane >= o) before += t; }
                before -= sum;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (before < left && left <= before + n[k]) { choice[0] = 255 - 4 * lane - k; choice[1] = left - before; }
                    before += n[k];
                }
            }
            __syncthreads();
            limit |= choice[0] << shift;
            left = choice[1];
        }
    }
    uint32_t n_gt = 0, n_eq = 0;
    each([&](int, uint32_t rank) __attribute__((always_inline)) {
        n_gt += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(rank > limit));
        n_eq += (uint32_t)__builtin_popcountll(__builtin_amdgcn_ballot_w64(rank == limit));
        asm volatile("" : "+s"(n_gt), "+s"(n_eq));
    });
    if (lane == 0) { above[wave] = n_gt; equal[wave] = n_eq; }
    __syncthreads();
    uint32_t at = 0, ties = 0;
    for (int w = 0; w < wave; ++w) { at += above[w]; ties += equal[w]; }
    at += ties < left ? ties : left;
    limit = (uint32_t)__builtin_amdgcn_readfirstlane((int)limit);
    int from = lane;
    asm volatile("" : "+s"(limit), "+v"(from));   // (comparisons and addresses are made again: those of above would fill the registers)
    // (eight times 64 positions side by side)
    constexpr int BATCH = HELD > 0 && HELD < 8 ? HELD : 8;
    auto write = [&](int k0, const uint32_t (&rank)[BATCH]) __attribute__((always_inline)) {
        uint32_t to[BATCH];
        float x[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            bool stays = rank[u] > limit && k0 + u < steps;
            unsigned long long g = __builtin_amdgcn_ballot_w64(stays);
            if (ties < left) {   // (the same for the whole wave, as what follows)
                const bool tie = rank[u] == limit && k0 + u < steps;
                const unsigned long long e = __builtin_amdgcn_ballot_w64(tie);
                if (e != 0) {
                    stays = stays || (tie && lanes_below(e, ties) < left);
                    g = __builtin_amdgcn_ballot_w64(stays);
                    ties += (uint32_t)__builtin_popcountll(e);
                }
            }
            to[u] = stays ? lanes_below(g, at) : ~0u;
            at += (uint32_t)__builtin_popcountll(g);
        }
        // (a rank says which number it was made from; those that stay in any case are read again)
        if (out) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) {
                x[u] = mass_of_rank(rank[u]);
                if (rank[u] == ~0u && to[u] != ~0u) x[u] = mass[p0 + 64 * (k0 + u) + from];
            }
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (to[u] == ~0u) continue;
            kept[to[u]] = p0 + 64 * (k0 + u) + from;
            if (out) out[to[u]] = x[u];
        }
    };
    if constexpr (HELD > 0) {
#pragma unroll
        for (int k0 = 0; k0 < HELD; k0 += BATCH) {
            if (k0 >= steps) break;   // (the same for the whole wave)
            uint32_t rank[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) rank[u] = held[k0 + u];
            write(k0, rank);
            __builtin_amdgcn_sched_barrier(0);
        }
    } else {
        for (int k0 = 0; k0 < steps; k0 += BATCH) {
            uint32_t rank[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; ++u) rank[u] = __float_as_uint(load(k0 + u));
#pragma unroll
            for (int u = 0; u < BATCH; ++u) rank[u] = rank_of(k0 + u, __uint_as_float(rank[u]));
            write(k0, rank);
        }
    }
}

struct MoveArgs {
    const void *src;
    void *dst;
    const int32_t *src_table, *dst_table, *kept;
    int32_t *dst_len;   // (device copy of the length)
    double turn[64];    // theta / (2 pi) of every rotary pair
    int32_t rotate, keep, n_layers, n_kv_heads, page_tokens;
};

constexpr int kMoveThreads = 512, kMovePages = 8;   // pages of 16 tokens at a time

// cos and sin of the turn by `moved` positions, the angle reduced in 64 bits.  ROUGH: by the hardware's functions of a turn, to about
// 2^-20, for keys that are rounded to bf16 behind it.
template <bool ROUGH>
__device__ __forceinline__ void turn_of(double turn, int moved, float &c, float &s)
{
    const double t = (double)moved * turn;
    const float f = (float)(t - rint(t));
    if (ROUGH) {
        c = __builtin_amdgcn_cosf(f);
        s = __builtin_amdgcn_sinf(f);
    } else sincospif(2.f * f, &s, &c);
}

// The cache in matrix-core order.  Block = (layer, head; keys or values; every gridDim.z-th group of eight pages): all that goes into the
// group is read before any of it is written, and a position never moves up, so a cache may be moved into itself with one block
// per layer, head and kind (gridDim.z = 1).  A line of the cache has eight keys' pieces or 16 dims of four values, so that every line with
// something that stays is read: of 65536 positions a quarter at random, 320 MB in 89 us (3.6 TB/s) for 134 MB that are kept; of 3584 two layers of 32
// heads, 150 MB in 40 us.   grid: (n_layers * n_kv_heads, 2, groups)
template <int DH>
__global__ __launch_bounds__(kMoveThreads) void cache_move_kernel(const MoveArgs a)
{
    const int tid = threadIdx.x, layer = blockIdx.x / a.n_kv_heads, head = blockIdx.x - layer * a.n_kv_heads, kind = blockIdx.y;
    if (blockIdx.x + blockIdx.y + blockIdx.z == 0 && tid == 0) *a.dst_len = a.keep;
    const int32_t *kept = a.kept + (size_t)blockIdx.x * a.keep;
    const int pages = (a.keep + 15) / 16;
    const bf16_t *src = (const bf16_t *)a.src;
    bf16_t *dst = (bf16_t *)a.dst;
    __shared__ int pos[kMovePages * 16], page[kMovePages * 16];
    for (int g = blockIdx.z; g * kMovePages < pages; g += gridDim.z) {
        const int first = g * kMovePages * 16;
        if (tid < kMovePages * 16) {
            const int i = first + tid;
            pos[tid] = i < a.keep ? kept[i] : -1;
            page[tid] = i < a.keep ? a.src_table[kept[i] >> 4] : 0;
        }
        __syncthreads();
        if (kind == 0) {
            // 16 bytes of a key and the 16 that they turn with
            constexpr int PAIRS = DH / 16, STEPS = kMovePages * 16 * PAIRS / kMoveThreads;
            uint4 lo[STEPS], hi[STEPS];
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int x = u * kMoveThreads + tid, t = x & 15, c = (x >> 4) % PAIRS, slot = (x >> 4) / PAIRS * 16 + t, p = pos[slot];
                lo[u] = hi[u] = make_uint4(0, 0, 0, 0);
                if (p < 0) continue;
                const bf16_t *from = src + kvf_base(page[slot], layer, a.n_layers, 0, head, a.n_kv_heads, DH);
                lo[u] = *(const uint4 *)(from + kf_elem(p & 15, 8 * c));
                hi[u] = *(const uint4 *)(from + kf_elem(p & 15, 8 * c + DH / 2));
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int x = u * kMoveThreads + tid, t = x & 15, c = (x >> 4) % PAIRS, slot = (x >> 4) / PAIRS * 16 + t, p = pos[slot];
                if (p < 0) continue;
                const int to = first + slot;
                if (a.rotate && p != to) {
                    uint32_t *l = &lo[u].x, *h = &hi[u].x;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        float r[2][2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float x0 = e ? __uint_as_float(l[w] & 0xffff0000u) : __uint_as_float(l[w] << 16);
                            const float x1 = e ? __uint_as_float(h[w] & 0xffff0000u) : __uint_as_float(h[w] << 16);
                            float cs, sn;
                            turn_of<true>(a.turn[8 * c + 2 * w + e], to - p, cs, sn);
                            r[0][e] = x0 * cs - x1 * sn;   // (the cache's own type is what there is room for)
                            r[1][e] = x1 * cs + x0 * sn;
                        }
                        l[w] = pack_bf16(r[0][0], r[0][1]);
                        h[w] = pack_bf16(r[1][0], r[1][1]);
                    }
                }
                bf16_t *put = dst + kvf_base(a.dst_table[to >> 4], layer, a.n_layers, 0, head, a.n_kv_heads, DH);
                *(uint4 *)(put + kf_elem(to & 15, 8 * c)) = lo[u];
                *(uint4 *)(put + kf_elem(to & 15, 8 * c + DH / 2)) = hi[u];
            }
        } else {
            // one dim of four tokens
            constexpr int UNITS = DH * 4, STEPS = kMovePages * UNITS / kMoveThreads;
            bf16_t v[STEPS][4];
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int x = u * kMoveThreads + tid, dim = (x & 15) + 16 * ((x >> 6) % (DH / 16)), slot = x / UNITS * 16 + ((x >> 4) & 3) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = pos[slot + e];
                    v[u][e] = p < 0 ? 0 : src[kvf_base(page[slot + e], layer, a.n_layers, 1, head, a.n_kv_heads, DH) + vf_elem(p & 15, dim)];
                }
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                const int x = u * kMoveThreads + tid, dim = (x & 15) + 16 * ((x >> 6) % (DH / 16)), slot = x / UNITS * 16 + ((x >> 4) & 3) * 4;
                if (pos[slot] < 0) continue;
                const int to = first + slot;
                bf16_t *put = dst + kvf_base(a.dst_table[to >> 4], layer, a.n_layers, 1, head, a.n_kv_heads, DH) + vf_elem(to & 15, dim);
                *(uint2 *)put = make_uint2((uint32_t)v[u][0] | ((uint32_t)v[u][1] << 16), (uint32_t)v[u][2] | ((uint32_t)v[u][3] << 16));
            }
        }
        __syncthreads();   // (the list is about to be replaced)
    }
}

// Caches in plain order: rows of [dim], whatever the page size.   grid: as above
template <typename KT, int DH>
__global__ __launch_bounds__(kMoveThreads) void cache_move_plain_kernel(const MoveArgs a)
{
    constexpr int PAIRS = DH / 2, TOKENS = kMovePages * 16, STEPS = TOKENS * PAIRS / kMoveThreads;
    const int tid = threadIdx.x, layer = blockIdx.x / a.n_kv_heads, head = blockIdx.x - layer * a.n_kv_heads, kind = blockIdx.y, pt = a.page_tokens;
    if (blockIdx.x + blockIdx.y + blockIdx.z == 0 && tid == 0) *a.dst_len = a.keep;
    const int32_t *kept = a.kept + (size_t)blockIdx.x * a.keep;
    const KT *src = (const KT *)a.src;
    KT *dst = (KT *)a.dst;
    __shared__ int pos[TOKENS];
    for (int g = blockIdx.z; g * TOKENS < a.keep; g += gridDim.z) {
        const int first = g * TOKENS;
        if (tid < TOKENS) pos[tid] = first + tid < a.keep ? kept[first + tid] : -1;
        __syncthreads();
        KT lo[STEPS], hi[STEPS];
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int x = u * kMoveThreads + tid, i = x % PAIRS, p = pos[x / PAIRS];
            lo[u] = hi[u] = KT(0);
            if (p < 0) continue;
            const KT *from = src + kv_offset(a.src_table[p / pt], layer, a.n_layers, kind, head, a.n_kv_heads, p % pt, pt, DH);
            lo[u] = from[i];
            hi[u] = from[i + PAIRS];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
            const int x = u * kMoveThreads + tid, i = x % PAIRS, p = pos[x / PAIRS], to = first + x / PAIRS;
            if (p < 0) continue;
            KT *put = dst + kv_offset(a.dst_table[to / pt], layer, a.n_layers, kind, head, a.n_kv_heads, to % pt, pt, DH);
            if (kind == 0 && a.rotate && p != to) {
                float cs, sn;
                turn_of<sizeof(KT) == 2>(a.turn[i], to - p, cs, sn);
                const float x0 = load_f32(&lo[u], 0), x1 = load_f32(&hi[u], 0);
                store_kv(put, i, x0 * cs - x1 * sn);
                store_kv(put, i + PAIRS, x1 * cs + x0 * sn);
            } else {
                put[i] = lo[u];
                put[i + PAIRS] = hi[u];
            }
        }
        __syncthreads();
    }
}

}  // namespace anpd
