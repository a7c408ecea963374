// Drawing tokens from logits, for gfx950.
//
//   a_i = (x_i - max x) / T,  w_i = exp a_i.  Tokens in order: larger logits first, equal ones by index.
//   K: the first top_k.  P: those of K before which less than top_p sum_K w has been summed.  M: w_i >= min_p.
//   kept = K, P and M together;  token = the lowest index i with sum_{j <= i, kept} w_j > u sum_kept w;  log p = a_token - log sum_kept w
//
// Sums.  Which token a random number falls on is decided by sums that are compared, so they are held in 64-bit integers: a weight is formed
// in 64 bits and rounded once to a multiple of 2^-shift of the largest, and then every sum is exact, whatever its order.  Histograms may
// be filled by atomics and rows divided among threads as one likes; the same inputs give the same token.
//
// Order.  The kept tokens are the first ones of an order, so they are told from the others by one logit and an index among its equals.
// That logit is found without sorting: a histogram of 2048 equal intervals says which one holds the border, which is divided again, until all logits in
// it are the same: three rounds at most in 2^33 of a range, two with a model's logits.
#pragma once
#include "anpd_layout.h"

namespace anpd {

constexpr int kSampleBins = 2048, kSampleHeld = 32;   // logits that a thread holds
constexpr int kSampleMaxVocab = 1 << 20;

struct SampleArgs {
    const void *logits;
    int64_t ld;
    const float *uniform;
    const float *temperatures, *top_ps, *min_ps;   // of each row, or NULL: those below
    const int32_t *top_ks;
    int32_t *token;
    float *logprob;   // may be NULL
    float temperature, top_p, min_p;
    int32_t top_k, rows, vocab, f32, wide, shift;
};

template <int THREADS>
struct SampleShared {
    static constexpr int kWaves = THREADS / 64, kChunks = kSampleMaxVocab / (4 * THREADS);
    unsigned long long bins[kSampleBins];       // weights, or counts
    unsigned long long segment[THREADS == 1024 ? kChunks * kWaves : kSampleHeld / 4 * kWaves];   // of 256 adjacent tokens: weights, or numbers of equal logits
    unsigned long long wave_sum[kWaves];
    float wave_lo[kWaves], wave_hi[kWaves];
    unsigned long long found[2];   // sum in front of what was looked for; all of it
    int at;
};

// A block's row.  HELD: its logits lie in registers; otherwise they are read again for each pass.
template <int THREADS, bool HELD>
struct Sampler {
    static constexpr int kWaves = THREADS / 64, kChunk = 4 * THREADS, kHeldChunks = kSampleHeld / 4;
    const SampleArgs &a;
    SampleShared<THREADS> &s;
    const int lane, wave, row;
    float held[HELD ? kHeldChunks : 1][4];
    bool infinite = false;   // some logit is: those alone have a weight
    double top = 0.0, per_t = 0.0, unit = 0.0;   // largest logit, 1 / T, 2^shift
    // kept: logits above `border`, and those equal to it up to index `last`
    float border = -INFINITY;
    int last = 0x7fffffff;

    __device__ __forceinline__ Sampler(const SampleArgs &args, SampleShared<THREADS> &shared)
        : a(args), s(shared), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), row(blockIdx.x) {}

    // Four adjacent logits; NaN and what lies behind the last token: minus infinity.
    __device__ __forceinline__ void load4(int i, float (&x)[4]) const
    {
        const size_t at = (size_t)row * a.ld + i;
        if (a.wide && i + 4 <= a.vocab) {
            if (a.f32) {
                const f32x4 v = *(const f32x4 *)((const float *)a.logits + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = v[e];
            } else {
                const uint2 v = *(const uint2 *)((const bf16_t *)a.logits + at);
                x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
                x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = i + e >= a.vocab ? -INFINITY : a.f32 ? ((const float *)a.logits)[at + e] : bf16_to_f32(((const bf16_t *)a.logits)[at + e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!(x[e] >= -INFINITY)) x[e] = -INFINITY;
            if (infinite) x[e] = x[e] == INFINITY ? 0.f : -INFINITY;
        }
    }
    __device__ __forceinline__ int index(int chunk) const { return chunk * kChunk + 4 * (int)threadIdx.x; }
    // f(chunk, first index, four logits) for all of the thread's
    template <typename F>
    __device__ __forceinline__ void each(F f)
    {
        if constexpr (HELD) {
#pragma unroll
            for (int c = 0; c < kHeldChunks; ++c) {
                if (c * kChunk >= a.vocab) break;   // (the same for all)
                f(c, index(c), held[c]);
            }
        } else {
            for (int c = 0; c * kChunk < a.vocab; ++c) {
                float x[4];
                load4(index(c), x);
                f(c, index(c), x);
            }
        }
    }

    __device__ __forceinline__ double weight(float x) const { return exp(((double)x - top) * per_t); }
    __device__ __forceinline__ unsigned long long units(double w) const { return (unsigned long long)(w * unit + 0.5); }

    __device__ __forceinline__ void reduce_range(float &lo, float &hi)
    {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) { lo = fminf(lo, __shfl_xor(lo, o, 64)); hi = fmaxf(hi, __shfl_xor(hi, o, 64)); }
        __syncthreads();
        if (lane == 0) { s.wave_lo[wave] = lo; s.wave_hi[wave] = hi; }
        __syncthreads();
        lo = s.wave_lo[0];
        hi = s.wave_hi[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) { lo = fminf(lo, s.wave_lo[w]); hi = fmaxf(hi, s.wave_hi[w]); }
    }
    static __device__ __forceinline__ unsigned long long wave_scan(unsigned long long v, int lane)   // inclusive
    {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned long long w = __shfl_up(v, o, 64);
            if (lane >= o) v += w;
        }
        return v;
    }
    // Of n numbers in LDS: the first whose sum with those before it reaches `goal(sum of all)` (at least 1).  Its place; found[] says the rest.
    template <typename Goal>
    __device__ __forceinline__ int find(const unsigned long long *v, int n, Goal goal)
    {
        const int each = (n + THREADS - 1) / THREADS, lo = (int)threadIdx.x * each, hi = lo + each < n ? lo + each : n;
        unsigned long long mine = 0;
        for (int i = lo; i < hi; ++i) mine += v[i];
        const unsigned long long to = wave_scan(mine, lane);
        if (lane == 63) s.wave_sum[wave] = to;
        __syncthreads();
        unsigned long long before = to - mine, all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += s.wave_sum[w];
            all += s.wave_sum[w];
        }
        const unsigned long long want = goal(all);
        if (before < want && before + mine >= want) {   // (one thread's)
            int i = lo;
            while (before + v[i] < want) before += v[i++];
            s.found[0] = before;
            s.found[1] = all;
            s.at = i;
        }
        __syncthreads();
        return s.at;
    }

    // Ends the kept ones where `goal(sum of all that are kept so far)` is reached by what `amount(x)` adds up to, in their order.
    template <typename Amount, typename Goal>
    __device__ __forceinline__ void cut(float lo, float hi, Amount amount, Goal goal)
    {
        unsigned long long want = 0;   // (from the first round on)
        bool first = true;
        for (;;) {
            for (int i = threadIdx.x; i < kSampleBins; i += THREADS) s.bins[i] = 0;
            __syncthreads();
            const double from = hi, per = lo < hi ? kSampleBins / ((double)hi - (double)lo) : 0.0;
            auto bin = [&](float x) __attribute__((always_inline)) {
                const int b = (int)((from - (double)x) * per);
                return b < kSampleBins ? b : kSampleBins - 1;
            };
            each([&](int, int i0, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x[e] >= lo && x[e] <= hi && (x[e] > border || (x[e] == border && i0 + e <= last))) atomicAdd(&s.bins[bin(x[e])], amount(x[e]));
            });
            __syncthreads();
            const int b = find(s.bins, kSampleBins, [&](unsigned long long all) { return first ? (want = goal(all)) : want; });
            const unsigned long long before = s.found[0];
            want -= before;
            first = false;
            float low = INFINITY, high = -INFINITY;
            each([&](int, int, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (x[e] >= lo && x[e] <= hi && bin(x[e]) == b) { low = fminf(low, x[e]); high = fmaxf(high, x[e]); }
            });
            reduce_range(low, high);
            lo = low;
            hi = high;
            if (lo == hi) break;
        }
        // all in it are equal: so many of them, by index
        const unsigned long long one = amount(lo), count = (want + one - 1) / one;
        const int end = last;
        each([&](int c, int i0, const float (&x)[4]) __attribute__((always_inline)) {
            unsigned long long n = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) n += __popcll(__builtin_amdgcn_ballot_w64(x[e] == lo && (lo > border || i0 + e <= end)));
            if (lane == 0) s.segment[c * kWaves + wave] = n;
        });
        __syncthreads();
        const int at = find(s.segment, segments(), [&](unsigned long long) { return count; });
        if (wave == 0) {
            const unsigned long long left = count - s.found[0];
            float x[4];
            load4(at * 256 + 4 * lane, x);
            unsigned long long n = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) n += x[e] == lo;
            unsigned long long to = wave_scan(n, lane) - n;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (x[e] == lo && ++to == left) s.at = at * 256 + 4 * lane + e;
        }
        __syncthreads();
        border = lo;
        last = s.at;
        __syncthreads();
    }
    __device__ __forceinline__ int segments() const { return (a.vocab + kChunk - 1) / kChunk * kWaves; }

    __device__ __forceinline__ void done(int token, float logprob) const
    {
        a.token[row] = token;
        if (a.logprob) a.logprob[row] = logprob;
    }

    __device__ __forceinline__ void draw()
    {
        if constexpr (HELD) {
#pragma unroll
            for (int c = 0; c < kHeldChunks; ++c) {
                if (c * kChunk >= a.vocab) break;
                load4(index(c), held[c]);
            }
        }
        float lo = INFINITY, hi = -INFINITY;
        unsigned long long valid = 0;
        each([&](int, int, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (x[e] > -INFINITY) { lo = fminf(lo, x[e]); ++valid; }
                hi = fmaxf(hi, x[e]);
            }
        });
        reduce_range(lo, hi);
        if (hi == -INFINITY) {   // no token
            if (threadIdx.x == 0) done(-1, __uint_as_float(0x7fc00000u));
            return;
        }
        if (hi == INFINITY) {
            infinite = true;
            valid = 0;
            if constexpr (HELD) {
#pragma unroll
                for (int c = 0; c < kHeldChunks; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) held[c][e] = c * kChunk < a.vocab && held[c][e] == INFINITY ? 0.f : -INFINITY;
            }
            each([&](int, int, const float (&x)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) valid += x[e] == 0.f;
            });
            lo = hi = 0.f;
        }
        const float temperature = a.temperatures ? a.temperatures[row] : a.temperature, top_p = a.top_ps ? a.top_ps[row] : a.top_p,
                    min_p = a.min_ps ? a.min_ps[row] : a.min_p;
        const int top_k = a.top_ks ? a.top_ks[row] : a.top_k;
        const bool greedy = !(temperature > 0.f);
        top = hi;
        per_t = 1.0 / (double)temperature;
        unit = (double)(1ull << a.shift);
        auto one = [](float) __attribute__((always_inline)) { return 1ull; };
        if (greedy) cut(hi, hi, one, [](unsigned long long) { return 1ull; });
        else {
            const unsigned long long upto = wave_scan(valid, lane);
            if (lane == 63) s.wave_sum[wave] = upto;
            __syncthreads();
            valid = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) valid += s.wave_sum[w];
            __syncthreads();
            if (top_k > 0 && (unsigned long long)top_k < valid) cut(lo, hi, one, [&](unsigned long long) { return (unsigned long long)top_k; });
            if (top_p < 1.f) {
                cut(border > lo ? border : lo, hi, [&](float x) __attribute__((always_inline)) { return units(weight(x)); }, [&](unsigned long long all) {
                    const double p = top_p > 0.f ? ceil((double)top_p * (double)all) : 0.0;
                    const unsigned long long want = p >= (double)all ? all : (unsigned long long)p;
                    return want > 0 ? want : 1ull;
                });
            }
        }
        const double floor_w = min_p > 0.f ? (min_p < 1.f ? (double)min_p : 1.0) : 0.0;
        auto kept = [&](float x, int i) __attribute__((always_inline)) {
            if (!(x > border || (x == border && i <= last)) || x == -INFINITY) return 0ull;
            if (greedy) return 1ull;
            const double w = weight(x);
            return w >= floor_w ? units(w) : 0ull;
        };
        each([&](int c, int i0, const float (&x)[4]) __attribute__((always_inline)) {
            unsigned long long n = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) n += kept(x[e], i0 + e);
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
            if (lane == 0) s.segment[c * kWaves + wave] = n;
        });
        __syncthreads();
        const float u = a.uniform[row];
        unsigned long long want = 0;
        const int at = find(s.segment, segments(), [&](unsigned long long all) {
            want = u > 0.f ? (u < 1.f ? (unsigned long long)((double)u * (double)all) : all) : 0;   // (a NaN: 0)
            want = want < all ? want + 1 : all;
            return want;
        });
        if (wave == 0) {
            const unsigned long long left = want - s.found[0];
            float x[4];
            load4(at * 256 + 4 * lane, x);
            unsigned long long n[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) { n[e] = kept(x[e], at * 256 + 4 * lane + e); sum += n[e]; }
            unsigned long long to = wave_scan(sum, lane) - sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (to < left && to + n[e] >= left)
                    done(at * 256 + 4 * lane + e, greedy ? 0.f : (float)(((double)x[e] - top) * per_t - log((double)s.found[1] / unit)));
                to += n[e];
            }
        }
    }
};

template <int THREADS, bool HELD>
__global__ __launch_bounds__(THREADS) void sample_kernel(const SampleArgs a)
{
    __shared__ SampleShared<THREADS> shared;
    Sampler<THREADS, HELD> sampler(a, shared);
    sampler.draw();
}

}  // namespace anpd
