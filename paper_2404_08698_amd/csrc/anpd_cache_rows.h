// Rows of keys and values into paged caches and back, for gfx950: rounded to the cache's type, or quantised to 8 bits.
//
//   8 bits, per position and head, keys and values apart:  s = max |x| / 127 in fp32,  code = 127 x / max |x| to the nearest, ties to even;  value = code s
//
// A wave has 16 positions of a sequence (those of a page, where pages are 16 long), one key / value head, keys or values: no 32-bit word of a cache is written by two
// waves, and its values, which lie key beside key, are turned around in the wave.  Into 8 bits and plain order bound by the bytes read and written: 3584 rows of 32 heads of 128 in
// bf16, into 8 bits 26 us (3.4 TB/s of what is read and written; back to back 22), back 15 (5.9 TB/s, from L2 in part); into fp32 in plain order 28 and back 27 (6.3 and 6.5);
// a row for each of 32 caches into 8 bits 6.2 and 4.5, a launch's length.  Into matrix-core order (bf16, pages of 16) bound by its accesses, which are 2 bytes each: 55 and 57 us (2.1 TB/s).
#pragma once
#include "anpd_cache_softmax.h"

namespace anpd {

enum CacheKind { kCacheF32, kCacheBf16, kCacheFragments, kCache8 };
constexpr int kRowsWaves = 4;

struct RowsArgs {
    SeqView seq[kAttnMaxSeqs];   // block0: first span of 16 positions
    void *k, *v;                 // the rows (read or written)
    int64_t ldk, ldv;
    int32_t layer, n_layers, n_kv_heads, page_tokens;
    int32_t wide;                // whether the rows may be moved 16 bytes at a time
    int32_t n_seq, n_spans;
};

// Eight dims of a row of type T.
template <typename T>
__device__ __forceinline__ void load_row8(const RowsArgs &a, const void *rows, size_t at, float (&x)[8])
{
    const T *p = (const T *)rows + at;
    if constexpr (std::is_same<T, float>::value) {
        if (a.wide) {
            const f32x4 u = *(const f32x4 *)p, v = *(const f32x4 *)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = u[i]; x[4 + i] = v[i]; }
            return;
        }
    } else if (a.wide) {
        const u32x4 u = *(const u32x4 *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = load_f32(p, (size_t)i);
}
template <typename T>
__device__ __forceinline__ void store_row8(const RowsArgs &a, void *rows, size_t at, const float (&x)[8])
{
    T *p = (T *)rows + at;
    if constexpr (std::is_same<T, float>::value) {
        if (a.wide) {
            *(f32x4 *)p = (f32x4){x[0], x[1], x[2], x[3]};
            *(f32x4 *)(p + 4) = (f32x4){x[4], x[5], x[6], x[7]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = x[i];
        }
    } else {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        if (a.wide) *(u32x4 *)p = w;
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) { p[2 * i] = (bf16_t)w[i]; p[2 * i + 1] = (bf16_t)(w[i] >> 16); }
        }
    }
}

// Four words of four bytes each <-> the same bytes the other way round.
__device__ __forceinline__ void transpose4(const uint32_t (&a)[4], uint32_t (&d)[4])
{
    const uint32_t x = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), y = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u);
    const uint32_t z = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u), w = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
    d[0] = __builtin_amdgcn_perm(y, x, 0x05040100u);
    d[1] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    d[2] = __builtin_amdgcn_perm(w, z, 0x05040100u);
    d[3] = __builtin_amdgcn_perm(w, z, 0x07060302u);
}

// Eight codes + 128, bytes side by side: 127 x / top to the nearest whole number, ties to even; per = 127 / top.  A product in 32 bits is off by 2^-16 at most, so it
// decides unless it lies next to the middle between two codes (or per is beyond 32 bits); there the quotient in 64 bits does: one that is not the middle
// is 2^-33 of it away, and the middle itself comes out exactly.
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], float top, float per)
{
    const float magic = 12582912.0f;   // (1.5 2^23: what is added to it is rounded to a whole number, which its lowest bits hold)
    uint32_t b[8];
    float far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = x[e] * per, k = t + magic;
        far = fmaxf(far, fabsf(t - (k - magic)));
        b[e] = __float_as_uint(k);
    }
    if (!(far < 0.5f - 0x1p-15f) || !(per < 0x1p120f)) {
        uint32_t near = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float t = x[e] * per;
            near |= !(fabsf(t - (t + magic - magic)) < 0.5f - 0x1p-15f) || !(per < 0x1p120f) ? 1u << e : 0u;
        }
        while (near) {   // (one of them, as a rule)
            const int e = __builtin_ctz(near);
            near &= near - 1;
            float v = x[0];
#pragma unroll
            for (int u = 1; u < 8; ++u) v = e == u ? x[u] : v;
            const uint32_t c = (uint32_t)(int)rint(127.0 * (double)v / (double)top);
#pragma unroll
            for (int u = 0; u < 8; ++u) b[u] = e == u ? c : b[u];
        }
    }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x00000400u), hi = __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x04000000u);
        w[h] = ((lo & 0xffffu) | (hi & 0xffff0000u)) ^ 0x80808080u;
    }
    return make_uint2(w[0], w[1]);
}

// What a wave of the kernels below is about.
struct Span {
    SeqView s;
    int first, from, to;   // position of the span, and which of its 16 are new rows
    int head, kind;        // keys 0, values 1
    __device__ __forceinline__ bool find(const RowsArgs &a)
    {
        const int64_t item = (int64_t)blockIdx.x * kRowsWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        kind = (int)(item % 2);
        head = (int)(item / 2 % a.n_kv_heads);
        const int64_t span = item / 2 / a.n_kv_heads;
        if (span >= a.n_spans) return false;
        int lo = 0, hi = a.n_seq - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.seq[mid].block0 <= span) lo = mid;
            else hi = mid - 1;
        }
        s = a.seq[lo];
        first = (s.pos0 / 16 + (int)(span - s.block0)) * 16;
        from = s.pos0 > first ? s.pos0 - first : 0;
        to = s.pos0 + s.n < first + 16 ? s.pos0 + s.n - first : 16;
        return true;
    }
};

// Plain and matrix-core order: eight dims of a position by each lane.
template <int KIND, int DH, bool STORE, typename T>
__device__ __forceinline__ void move_rows(const RowsArgs &a, const Span &w)
{
    constexpr int LANES = DH / 8;
    const int lane = threadIdx.x & 63, dim = lane % LANES * 8;
    void *rows = w.kind ? a.v : a.k;
    const int64_t ld = w.kind ? a.ldv : a.ldk;
    for (int t = lane / LANES; t < 16; t += 64 / LANES) {
        if (t < w.from || t >= w.to) continue;
        const int p = w.first + t;
        const size_t at = (size_t)(w.s.row0 + p - w.s.pos0) * ld + (size_t)w.head * DH + dim;
        const int page = w.s.table[p / a.page_tokens];
        float x[8];
        if (STORE) load_row8<T>(a, rows, at, x);
        if constexpr (KIND == kCacheFragments) {
            bf16_t *to = (bf16_t *)w.s.pool + kvf_base(page, a.layer, a.n_layers, w.kind, w.head, a.n_kv_heads, DH);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                bf16_t *e = to + (w.kind ? vf_elem(t, dim + i) : kf_elem(t, dim + i));
                if (STORE) *e = (bf16_t)pack_bf16(x[i], 0.f);
                else x[i] = bf16_to_f32(*e);
            }
        } else {
            typedef typename std::conditional<KIND == kCacheF32, float, bf16_t>::type KT;
            KT *to = (KT *)w.s.pool + kv_offset(page, a.layer, a.n_layers, w.kind, w.head, a.n_kv_heads, p % a.page_tokens, a.page_tokens, DH) + dim;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (KIND == kCacheF32) { if (STORE) to[i] = x[i]; else x[i] = to[i]; }
                else { if (STORE) to[i] = (bf16_t)pack_bf16(x[i], 0.f); else x[i] = bf16_to_f32(to[i]); }
            }
        }
        if (!STORE) store_row8<T>(a, rows, at, x);
    }
}

// 8 bits.  turn: LDS of the wave, [position][dim].
template <int DH, typename T>
__device__ __forceinline__ void quantise(const RowsArgs &a, const Span &w, uint32_t (&turn)[16][DH / 4])
{
    constexpr int LANES = DH / 8, STEP = 64 / LANES;
    const int lane = threadIdx.x & 63, dim = lane % LANES * 8;
    const void *rows = w.kind ? a.v : a.k;
    const int64_t ld = w.kind ? a.ldv : a.ldk;
    char *block = (char *)w.s.pool + kv8_base(w.s.table[w.first / 16], a.layer, a.n_layers, w.kind, w.head, a.n_kv_heads, DH);
    float *scales = (float *)(block + 16 * DH);
    float x[16 / STEP][8];
    // (all requested before the first is looked at; positions that are not new read a new one's row again)
#pragma unroll
    for (int i = 0; i < 16 / STEP; ++i) {
        const int t = i * STEP + lane / LANES, near = t < w.from ? w.from : t < w.to ? t : w.to - 1;
        load_row8<T>(a, rows, (size_t)(w.s.row0 + w.first + near - w.s.pos0) * ld + (size_t)w.head * DH + dim, x[i]);
    }
#pragma unroll
    for (int i = 0; i < 16 / STEP; ++i) {
        const int t = i * STEP + lane / LANES;
        if (i * STEP >= w.to || (i + 1) * STEP <= w.from) continue;   // (the same for the wave)
        uint32_t bits = 0;   // (as whole numbers: infinities and NaN are above all others)
#pragma unroll
        for (int e = 0; e < 8; ++e) { const uint32_t b = __float_as_uint(x[i][e]) & 0x7fffffffu; bits = b > bits ? b : bits; }
#pragma unroll
        for (int o = 1; o < LANES; o <<= 1) { const uint32_t b = (uint32_t)__shfl_xor((int)bits, o, 64); bits = b > bits ? b : bits; }
        const float top = __uint_as_float(bits), per = 127.0f / top;
        const bool finite = bits < 0x7f800000u;
        uint2 c = make_uint2(0x80808080u, 0x80808080u);
        if (finite && bits != 0) c = codes_of(x[i], top, per);
        if (t >= w.from && t < w.to) {
            if (lane % LANES == 0) scales[t] = finite ? top / 127.0f : __uint_as_float(0x7fc00000u);
            if (w.kind == 0) *(uint2 *)(block + k8_elem(t, dim)) = c;
        }
        if (w.kind == 1) *(uint2 *)&turn[t][dim / 4] = c;
    }
    if (w.kind == 0) return;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // four dims of the eight positions of a half
    if (lane >= DH / 2) return;
    const int half = lane / (DH / 4), quad = lane % (DH / 4);
    uint32_t out[2][4];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        uint32_t in[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) in[t] = turn[8 * g + 4 * half + t][quad];
        transpose4(in, out[g]);
    }
    char *to = block + v8_elem(4 * half, 4 * quad);
    if (w.from == 0 && w.to == 16) {
        *(u32x4 *)to = (u32x4){out[0][0], out[1][0], out[0][1], out[1][1]};
        *(u32x4 *)(to + 16) = (u32x4){out[0][2], out[1][2], out[0][3], out[1][3]};
        return;
    }
#pragma unroll
    for (int g = 0; g < 2; ++g)
        for (int t = 0; t < 4; ++t) {
            const int p = 8 * g + 4 * half + t;
            if (p < w.from || p >= w.to) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) to[8 * e + 4 * g + t] = (char)(out[g][e] >> (8 * t));
        }
}
template <int DH, typename T>
__device__ __forceinline__ void read_back(const RowsArgs &a, const Span &w, uint32_t (&turn)[16][DH / 4])
{
    constexpr int LANES = DH / 8, STEP = 64 / LANES;
    const int lane = threadIdx.x & 63, dim = lane % LANES * 8;
    void *rows = w.kind ? a.v : a.k;
    const int64_t ld = w.kind ? a.ldv : a.ldk;
    const char *block = (const char *)w.s.pool + kv8_base(w.s.table[w.first / 16], a.layer, a.n_layers, w.kind, w.head, a.n_kv_heads, DH);
    const float *scales = (const float *)(block + 16 * DH);
    if (w.kind == 1) {
        if (lane < DH / 2) {
            const int half = lane / (DH / 4), quad = lane % (DH / 4);
            const u32x4 *from = (const u32x4 *)(block + v8_elem(4 * half, 4 * quad));
            const u32x4 u = from[0], v = from[1];
            const uint32_t in[2][4] = {{u[0], u[2], v[0], v[2]}, {u[1], u[3], v[1], v[3]}};
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                uint32_t out[4];
                transpose4(in[g], out);
#pragma unroll
                for (int t = 0; t < 4; ++t) turn[8 * g + 4 * half + t][quad] = out[t];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int i = 0; i < 16 / STEP; ++i) {
        const int t = i * STEP + lane / LANES;
        if (t < w.from || t >= w.to) continue;
        const uint2 c = w.kind ? *(const uint2 *)&turn[t][dim / 4] : *(const uint2 *)(block + k8_elem(t, dim));
        const float s = scales[t];
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)((int)((e < 4 ? c.x : c.y) >> (8 * (e & 3)) & 0xffu) - 128) * s;
        store_row8<T>(a, rows, (size_t)(w.s.row0 + w.first + t - w.s.pos0) * ld + (size_t)w.head * DH + dim, x);
    }
}

// grid: n_spans * n_kv_heads * 2 waves, four to a block
template <int KIND, int DH, bool STORE, typename T>
__global__ __launch_bounds__(64 * kRowsWaves) void cache_rows_kernel(const RowsArgs a)
{
    Span w;
    if (!w.find(a)) return;
    if constexpr (KIND == kCache8) {
        __shared__ uint32_t turn[kRowsWaves][16][DH / 4];
        if (STORE) quantise<DH, T>(a, w, turn[threadIdx.x >> 6]);
        else read_back<DH, T>(a, w, turn[threadIdx.x >> 6]);
    } else move_rows<KIND, DH, STORE, T>(a, w);
}

// ------------------------------------------------------------------ the accepted rows move together
//
// Rows slot[0] < slot[1] < ... behind the committed positions move to the places behind these, in all layers.  A thread has a dim of all
// of them and never writes where it still has to read (slot[i] >= i), so a row may move into any place before it.
// grid: (n_layers * n_kv_heads, keys | values), DH threads
struct CommitArgs {
    char *pool;
    const int32_t *table;
    int32_t len, n, n_layers, n_kv_heads, page_tokens;
    uint8_t slot[kTreeRows];
};
template <int KIND, int DH>
__global__ __launch_bounds__(DH) void cache_commit_kernel(const CommitArgs a)
{
    typedef typename std::conditional<KIND == kCacheF32, float, typename std::conditional<KIND == kCache8, char, bf16_t>::type>::type KT;
    const int head = blockIdx.x % a.n_kv_heads, layer = blockIdx.x / a.n_kv_heads, kind = blockIdx.y, dim = threadIdx.x;
    auto element = [&](int p) __attribute__((always_inline)) -> KT * {
        const int page = a.table[p / a.page_tokens], t = p % a.page_tokens;
        if constexpr (KIND == kCache8) return a.pool + kv8_base(page, layer, a.n_layers, kind, head, a.n_kv_heads, DH) + (kind ? v8_elem(t, dim) : k8_elem(t, dim));
        else if constexpr (KIND == kCacheFragments) return (KT *)a.pool + kvf_base(page, layer, a.n_layers, kind, head, a.n_kv_heads, DH) + (kind ? vf_elem(t, dim) : kf_elem(t, dim));
        else return (KT *)a.pool + kv_offset(page, layer, a.n_layers, kind, head, a.n_kv_heads, t, a.page_tokens, DH) + dim;
    };
    constexpr int EACH = 8;
    for (int i0 = 0; i0 < a.n; i0 += EACH) {
        KT x[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i0 + i < a.n) x[i] = *element(a.len + a.slot[i0 + i]);
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i0 + i < a.n) *element(a.len + i0 + i) = x[i];
    }
    if constexpr (KIND == kCache8) {
        if (dim > 0) return;
        auto scale = [&](int p) { return (float *)(a.pool + kv8_base(a.table[p / 16], layer, a.n_layers, kind, head, a.n_kv_heads, DH) + 16 * DH) + p % 16; };
        for (int i = 0; i < a.n; ++i) *scale(a.len + i) = *scale(a.len + a.slot[i]);
    }
}

}  // namespace anpd
