// Drawing tokens from logits, for gfx950.
//
//   a_i = (x_i - max x) / T,  w_i = exp a_i.  Tokens in order: larger logits first, equal ones by index.
//   K: the first top_k.  P: those of K before which less than top_p sum_K w has been summed.  M: w_i >= min_p.
//   kept = K, P and M together;  token = the lowest index i with sum_{j <= i, kept} w_j > u sum_kept w;  log p = a_token - log sum_kept w
//
// Sums.  Which token a random number falls on is decided by sums that are compared, so weights are formed in 64 bits and rounded once to whole multiples of
// 2^-shift of the largest, whose sums are exact in any order: histograms may be filled by atomics.  shift is 51, or what keeps a row's sum below 2^62: 47 for 32000 tokens, 45
// for 131072, 42 for 2^20; a sum is off by a step for each token at most (half of one in a slice's, half in the row's).  Sums of different slices of a row are joined in
// 64-bit floating point, in the slices' order: the same inputs give the same token.
//
// Order.  The kept tokens are the first ones of an order, so they are told from the others by one logit and an index among its equals (the border).  It is
// found without sorting: a histogram over intervals of logits, the same ones for all slices, says which interval holds the border; its few logits are compared
// with one another.  Only where they are many, the interval is divided again, until all in it are the same.
//
// Two launches: a block for each slice of 4096 or 16384 logits (its largest one, its histogram), and a block for each row, which joins them, collects the logits
// around the border and draws: it reads the row once more, but forms weights of a single slice only.  The weights of a row, 24 instructions of 64 bits for each (15 with a table),
// are what one compute unit would be busy with (32000 logits: 12 us of 51 in a form of one block per row; 64 rows of 131072: 190).  Rows of up to two slices: one launch.
// A row of 32000 in fp32, top_k 50, top_p 0.95: slices 5.0 us, row 14.5; 17 rows, top_p 0.9: 5.9 and 18.5; 64 rows of 131072 in bf16: 16 (1.0 TB/s) and 28.  The row's
// block is bound by neither bytes nor instructions but by its steps, each of which waits for the one before: barriers of 16 waves, trips to memory, sums over lanes.
#pragma once
#include <type_traits>

#include "anpd_layout.h"

namespace anpd {

constexpr int kSliceLogits = 16;      // of a thread
constexpr int kSampleBins = 1024;
constexpr int kBinsPerNat = 64;        // intervals to a factor of e between weights
constexpr int kSampleFew = 512;        // logits that are compared with one another
constexpr int kSampleMaxVocab = 1 << 20, kMaxSlices = 64;
constexpr int kRowThreads = 1024, kFusedSlices = 2;
// Slices of 4096 logits, which leave a block of 256 threads 16 for each; of 16384 for vocabularies above 65536, whose histograms would be more to join than
// there is to read.
__host__ __device__ constexpr int slice_shift(int vocab) { return vocab <= 65536 ? 12 : 14; }

typedef unsigned long long whole_t;

// What is known of a slice.
struct Slice {
    whole_t all;      // its weights' sum (of its own largest), or the number of its logits
    float most;       // largest logit
    int32_t unused;
    whole_t bins[kSampleBins];
};

struct SampleArgs {
    const void *logits;
    int64_t ld;
    const float *uniform;
    const float *temperatures, *top_ps, *min_ps;   // of each row, or NULL: those below
    const int32_t *top_ks;
    int32_t *token;
    float *logprob;   // may be NULL
    Slice *slices;    // [rows][n_slices]
    float temperature, top_p, min_p;
    int32_t top_k, vocab, n_slices, slice_shift, f32, wide, shift;
};

// A row's rules.
struct RowRules {
    float temperature, top_p, min_p;
    int top_k;   // 0: all
    bool greedy;
    __device__ __forceinline__ RowRules(const SampleArgs &a, int row)
    {
        temperature = a.temperatures ? a.temperatures[row] : a.temperature;
        top_p = a.top_ps ? a.top_ps[row] : a.top_p;
        min_p = a.min_ps ? a.min_ps[row] : a.min_p;
        top_k = a.top_ks ? a.top_ks[row] : a.top_k;
        greedy = !(temperature > 0.f);
        if (greedy) { top_k = 1; temperature = 1.f; }   // (the first of the order)
        temperature = fminf(temperature, 3.4028234e38f);
        if (top_k < 0 || top_k >= a.vocab) top_k = 0;
    }
};

// ------------------------------------------------------------------ numbers

// 2^z to the nearest whole number, z <= 51: Taylor's sum to the power of 11 around a whole power (off by 2^-47 of the value at most), the power added to
// its exponent, the rounding by a sum with 2^52.
__device__ __forceinline__ whole_t whole_exp2(double z)
{
    z = fmax(z, -2.0);   // (rounds to 0)
    const double magic = 0x1.8p52, n = z + magic, t = (z - (n - magic)) * 0.693147180559945309417232;
    double p = 1.0 / 39916800.0;
    p = fma(p, t, 1.0 / 3628800.0);
    p = fma(p, t, 1.0 / 362880.0);
    p = fma(p, t, 1.0 / 40320.0);
    p = fma(p, t, 1.0 / 5040.0);
    p = fma(p, t, 1.0 / 720.0);
    p = fma(p, t, 1.0 / 120.0);
    p = fma(p, t, 1.0 / 24.0);
    p = fma(p, t, 1.0 / 6.0);
    p = fma(p, t, 0.5);
    p = fma(p, t, 1.0);
    p = fma(p, t, 1.0);
    const whole_t power = (whole_t)__double_as_longlong(p) + ((whole_t)(uint32_t)__double_as_longlong(n) << 52);
    return (whole_t)__double_as_longlong(__longlong_as_double((long long)power) + 0x1p52) & 0xfffffffffffffull;
}

// The same with a table of 2^(j / 128) at hand (LDS): Taylor's sum to the power of 4 around one of its entries, for the many weights of a slice: 15
// instructions of 64 bits, which take 8 cycles each, instead of 23.
constexpr int kPowers = 128;
__device__ __forceinline__ whole_t whole_exp2(double z, const double *powers)
{
    z = fmax(z, -2.0);
    const double magic = 0x1.8p52 / kPowers, n = z + magic, t = (z - (n - magic)) * 0.693147180559945309417232;
    const uint32_t parts = (uint32_t)__double_as_longlong(n);
    double p = fma(1.0 / 24.0, t, 1.0 / 6.0);
    p = fma(p, t, 0.5);
    p = fma(p, t, 1.0);
    p = fma(p, t, 1.0) * powers[parts % kPowers];
    const whole_t power = (whole_t)__double_as_longlong(p) + ((whole_t)(parts / kPowers) << 52);
    return (whole_t)__double_as_longlong(__longlong_as_double((long long)power) + 0x1p52) & 0xfffffffffffffull;
}

// Weights relative to `top`, and intervals of logits (any ascending function will do, so it is one of 32 bits); per: log2(e) / T.
struct Scale {
    double top, per, shift;
    float bins, first;   // intervals to a logit; the top's interval among all there are
    __device__ __forceinline__ Scale(float most, float temperature, int shift_by) : top(most), per(1.44269504088896340735992 / (double)temperature), shift(shift_by),
                                                                                    bins(fminf((float)kBinsPerNat / temperature, 0x1p120f)) { first = interval(most); }
    __device__ __forceinline__ whole_t weight(float x) const { return whole_exp2(fma((double)x - top, per, shift)); }   // (-infinity: 0)
    __device__ __forceinline__ whole_t weight(float x, const double *powers) const { return whole_exp2(fma((double)x - top, per, shift), powers); }
    __device__ __forceinline__ float interval(float x) const { return floorf(fminf(fmaxf(x * bins, -0x1p22f), 0x1p22f)); }
    // intervals below the top's, the last one for all that lie behind
    __device__ __forceinline__ int bin(float x) const { return (int)fminf(first - interval(x), (float)(kSampleBins - 1)); }
};

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lanes_before(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T add_before(T v)
{
    if constexpr (sizeof(T) == 4) return v + __builtin_bit_cast(T, lanes_before<CTRL, ROWS>(__builtin_bit_cast(uint32_t, v)));
    else {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        return v + __builtin_bit_cast(T, ((uint64_t)lanes_before<CTRL, ROWS>((uint32_t)(u >> 32)) << 32) | lanes_before<CTRL, ROWS>((uint32_t)u));
    }
}
// Sum over this lane and those before it (shifts within rows of 16 lanes, then rows take over the last lane of those before).
template <typename T>
__device__ __forceinline__ T wave_scan(T v)
{
    v = add_before<0x111, 0xf>(v);
    v = add_before<0x112, 0xf>(v);
    v = add_before<0x114, 0xf>(v);
    v = add_before<0x118, 0xf>(v);
    v = add_before<0x142, 0xa>(v);
    return add_before<0x143, 0xc>(v);
}
template <int CTRL>
__device__ __forceinline__ float max_before(float v) { return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, 0xf, 0xf, false))); }
__device__ __forceinline__ float wave_max(float v)
{
    v = max_before<0x111>(v);
    v = max_before<0x112>(v);
    v = max_before<0x114>(v);
    v = max_before<0x118>(v);
    v = max_before<0x142>(v);
    v = max_before<0x143>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// ------------------------------------------------------------------ slices

// NaN: minus infinity.  infinite: logits that are plus infinity are 0, and all there is.
__device__ __forceinline__ float as_logit(float x, bool infinite)
{
    if (infinite) return x == INFINITY ? 0.f : -INFINITY;
    return x >= -INFINITY ? x : -INFINITY;
}
// Four adjacent logits that are all there, as they come.
template <typename T>
struct Four {
    typename std::conditional<std::is_same<T, float>::value, f32x4, uint2>::type v;
    __device__ __forceinline__ void load(const T *p) { v = *(const decltype(v) *)p; }
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (std::is_same<T, float>::value) return v[e];
        else return __uint_as_float(e & 1 ? (e < 2 ? v.x : v.y) & 0xffff0000u : (e < 2 ? v.x : v.y) << 16);
    }
};
// Four adjacent logits from place i on; behind the last one: minus infinity.
template <typename T>
__device__ __forceinline__ void load4(const SampleArgs &a, const T *of_row, int i, bool infinite, float (&x)[4])
{
    if (a.wide && i + 4 <= a.vocab) {
        Four<T> v;
        v.load(of_row + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = i + e < a.vocab ? load_f32(of_row, (size_t)(i + e)) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = as_logit(x[e], infinite);
}

// A slice's largest logit, and a histogram of its weights (where top_k is given: of its logits).  out: global memory or LDS.
template <int THREADS>
struct SliceShared {
    whole_t bins[kSampleBins], sum[THREADS / 64];
    double powers[kPowers];
    float most[THREADS / 64];
};
template <typename T, int THREADS, int EACH>
__device__ __forceinline__ void look_at_slice(const SampleArgs &a, const RowRules &rules, const T *of_row, int slice, SliceShared<THREADS> &s, Slice *out)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float x[EACH][4];
#pragma unroll
    for (int c = 0; c < EACH; ++c) load4<T>(a, of_row, slice * (4 * EACH * THREADS) + 4 * (c * THREADS + (int)threadIdx.x), false, x[c]);
    float most = -INFINITY;
#pragma unroll
    for (int c = 0; c < EACH; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, x[c][e]);
    for (int i = threadIdx.x; i < kSampleBins; i += THREADS) s.bins[i] = 0;
    if (threadIdx.x < kPowers) s.powers[threadIdx.x] = exp2((double)threadIdx.x / kPowers);
    most = wave_max(most);
    if (lane == 0) s.most[wave] = most;
    __syncthreads();
    most = s.most[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) most = fmaxf(most, s.most[i]);
    whole_t sum = 0;
    if (most > -INFINITY) {
        const bool infinite = most == INFINITY;
        const Scale scale(infinite ? 0.f : most, rules.temperature, a.shift);
#pragma unroll
        for (int c = 0; c < EACH; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = infinite ? (x[c][e] == INFINITY ? 0.f : -INFINITY) : x[c][e];
                if (!(v > -INFINITY)) continue;
                const whole_t m = rules.top_k ? 1 : scale.weight(v, s.powers);
                sum += m;
                const int b = scale.bin(v);
                if (b < kSampleBins - 1 && m != 0) atomicAdd(&s.bins[b], m);   // (most logits of a peaked row lie in the last one, which nobody asks for)
            }
    }
    sum = wave_scan(sum);
    if (lane == 63) s.sum[wave] = sum;
    __syncthreads();
    for (int i = threadIdx.x; i < kSampleBins; i += THREADS) out->bins[i] = s.bins[i];
    if (threadIdx.x == 0) {
        whole_t all = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) all += s.sum[i];
        out->all = all;
        out->most = most;
    }
    __syncthreads();
}

// grid: (n_slices, rows)
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_slices_kernel(const SampleArgs a)
{
    __shared__ SliceShared<THREADS> shared;
    const int slice = blockIdx.x, row = blockIdx.y;
    look_at_slice<T, THREADS, kSliceLogits / 4>(a, RowRules(a, row), (const T *)a.logits + (size_t)row * a.ld, slice, shared, a.slices + (size_t)row * a.n_slices + slice);
}

// ------------------------------------------------------------------ rows

struct RowShared {
    static constexpr int kWaves = kRowThreads / 64;
    whole_t bins[kSampleBins];
    whole_t few_amount[kSampleFew], few_before[kSampleFew], few_below[kSampleFew];
    float few[kSampleFew];
    int few_at[kSampleFew], few_rank[kSampleFew];
    double factor[kMaxSlices];         // of a slice's weights: its largest logit's, of the row's
    int later[kMaxSlices];             // intervals from the row's largest logit to the slice's
    whole_t more[kMaxSlices];          // what the interval of the border adds to a slice's kept weights
    double kept[kMaxSlices];
    double part[kWaves];
    whole_t whole_part[kWaves];
    float most[kWaves];
    double before, all;
    whole_t whole_before, total;
    int at, place, count, found, found_at[kRowThreads];   // (found: those that may be in an interval)
    float border;
};

template <typename T>
struct RowSampler {
    static constexpr int kWaves = RowShared::kWaves;
    const SampleArgs &a;
    RowShared &s;
    const Slice *slices;
    const T *of_row;
    const RowRules rules;
    const int lane, wave, row;
    bool infinite;
    Scale scale;
    // kept: logits above `border`, and those equal to it up to index `last`
    float border = -INFINITY;
    int last = 0x7fffffff;

    __device__ __forceinline__ RowSampler(const SampleArgs &args, RowShared &shared, const Slice *of, const RowRules &r, int at, float most)
        : a(args), s(shared), slices(of), of_row((const T *)args.logits + (size_t)at * args.ld), rules(r), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), row(at), infinite(most == INFINITY),
          scale(most == INFINITY ? 0.f : most, r.temperature, args.shift) {}

    // f(logit, index) for the logits from low to high.
    template <typename F>
    __device__ __forceinline__ void sweep(float low, float high, F f) const
    {
#pragma unroll 4
        for (int i = threadIdx.x; i < a.vocab; i += kRowThreads) {
            const float v = as_logit(load_f32(of_row, (size_t)i), infinite);
            if (v >= low && v <= high && v > -INFINITY) f(v, i);
        }
    }
    // found(index) for the logits from low to high and no others, but that infinities and NaN may be missed; rows that may be read four logits at a time.  A thread
    // compares 32 at a time, the next ones requested before.
    static constexpr int kSweep = 32 * kRowThreads;
    __device__ __forceinline__ void request(int c, Four<T> (&x)[8]) const
    {
        // (a vocabulary's last logits, up to three, are left for the end; behind it the first ones of the row, for nothing)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = c + 4 * (u * kRowThreads + (int)threadIdx.x);
            x[u].load(of_row + (i + 4 <= a.vocab ? i : 0));
        }
    }
    template <typename F>
    __device__ __forceinline__ void sweep_wide(float low, float high, F found) const
    {
        Four<T> x[8];
        request(0, x);
#pragma unroll 1
        for (int c = 0; c < a.vocab; c += kSweep) {
            uint32_t hit = 0;
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) hit |= x[u][e] >= low && x[u][e] <= high ? 1u << (4 * u + e) : 0u;
            if (c + kSweep < a.vocab) request(c + kSweep, x);
            const int left = (a.vocab & ~3) - c - 4 * (int)threadIdx.x, fours = left <= 0 ? 0 : (left + 4 * kRowThreads - 1) / (4 * kRowThreads);
            hit = fours >= 8 ? hit : hit & ((1u << (4 * fours)) - 1);
            while (hit) {
                const int bit = __builtin_ctz(hit);
                hit &= hit - 1;
                found(c + (bit >> 2) * 4 * kRowThreads + 4 * (int)threadIdx.x + (bit & 3));
            }
        }
        if ((int)threadIdx.x < (a.vocab & 3)) found((a.vocab & ~3) + (int)threadIdx.x);   // (to be looked at)
    }
    __device__ __forceinline__ bool inside(float v, int i) const { return v > border || (v == border && i <= last && v > -INFINITY); }

    // The first of kSampleBins numbers, one for each thread, whose sum with those before it reaches `want` (none: the last); before: their sum.  One that is above 0: sums of
    // 64-bit floating point are formed in another order for every lane, so that a 0 may come out above what lies before it.
    template <typename N>
    __device__ __forceinline__ int first_to_reach(N mine, N want, N &before)
    {
        static_assert(kSampleBins == kRowThreads, "a number for each thread");
        constexpr bool WHOLE = std::is_same<N, whole_t>::value;
        N *parts = (N *)(WHOLE ? (void *)s.whole_part : (void *)s.part), *prev = (N *)(WHOLE ? (void *)&s.whole_before : (void *)&s.before);
        const N upto = wave_scan(mine);
        if (lane == 63) parts[wave] = upto;
        __syncthreads();
        N first = 0, now = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            if (i == wave) first = now;
            now += parts[i];
        }
        const whole_t some = __builtin_amdgcn_ballot_w64(mine > 0), reach = some & __builtin_amdgcn_ballot_w64(first + upto >= want);
        const bool here = first < want && first + parts[wave] >= want;   // (one wave's: the next one's first is this sum; it has numbers above 0)
        if (here ? lane == (reach ? __builtin_ctzll(reach) : 63 - __builtin_clzll(some | 1)) : now < want && threadIdx.x == kRowThreads - 1) {
            s.at = threadIdx.x;
            *prev = first + (upto - mine);
        }
        __syncthreads();
        before = *prev;
        const int at = s.at;
        __syncthreads();
        return at;
    }

    // ---- the border, among the logits lo .. hi (of those that are kept so far): where `want` is reached by weights (MASS) or by numbers
    struct Intervals {
        double from, per;
        __device__ __forceinline__ Intervals(float lo, float hi) : from(hi), per(lo < hi ? kSampleBins / ((double)hi - (double)lo) : 0.0) {}
        __device__ __forceinline__ int of(float v) const
        {
            const int b = (int)((from - (double)v) * per);
            return b < kSampleBins ? b : kSampleBins - 1;
        }
    };
    template <bool MASS>
    __device__ __forceinline__ whole_t amount(float v) const { return MASS ? scale.weight(v) : 1; }

    // Logits that are certainly not in interval b are outside low .. high.  (At temperatures near the largest number, intervals end beyond it, and the product with a
    // logit just below 0 may be below the smallest one, which makes it 0.)
    struct Interval {
        float low, high;
        __device__ __forceinline__ Interval(const Scale &scale, int b)
        {
            constexpr float most = 3.4028234e38f;
            const float at = scale.first - (float)b, lo = fminf(fmaxf(at / scale.bins, -most), most), hi = fminf(fmaxf((at + 1.f) / scale.bins, -most), most);
            low = lo - fabsf(lo) * 0x1p-20f - 0x1p-149f / scale.bins;
            high = hi + fabsf(hi) * 0x1p-20f;
            if (b == kSampleBins - 1 || !(fabsf(at) < 0x1p21f)) low = -INFINITY;
            if (!(fabsf(at) < 0x1p21f)) high = INFINITY;   // (where the numbers of intervals end)
        }
    };
    // Those of the row from low to high that `which` names: into `few` as far as they fit; their number, and, if they do not fit, smallest and largest.
    template <typename Which>
    __device__ __forceinline__ int collect(float low, float high, Which which, float &lo, float &hi)
    {
        __syncthreads();
        if (threadIdx.x == 0) s.count = s.found = 0;
        __syncthreads();
        int m = kSampleFew + 1;
        if (a.wide && !infinite && a.vocab >= 4) {
            // (which ones first; their logits are read again side by side)
            sweep_wide(low, high, [&](int i) __attribute__((always_inline)) {
                const int at = atomicAdd(&s.found, 1);
                if (at < kRowThreads) s.found_at[at] = i;
            });
            __syncthreads();
            const int n = s.found;
            if (n <= kRowThreads) {
                if ((int)threadIdx.x < n) {
                    const int i = s.found_at[threadIdx.x];
                    const float v = load_f32(of_row, (size_t)i);
                    if (v >= low && v <= high && v > -INFINITY && which(v, i)) {
                        const int at = atomicAdd(&s.count, 1);
                        if (at < kSampleFew) { s.few[at] = v; s.few_at[at] = i; }
                    }
                }
                __syncthreads();
                m = s.count;
                if (m <= kSampleFew) return m;
                __syncthreads();
                if (threadIdx.x == 0) s.count = 0;
                __syncthreads();
            }
        }
        float least = INFINITY, most = -INFINITY;
        sweep(low, high, [&](float v, int i) __attribute__((always_inline)) {
            if (!which(v, i)) return;
            const int at = atomicAdd(&s.count, 1);
            if (at < kSampleFew) { s.few[at] = v; s.few_at[at] = i; }
            least = fminf(least, v);
            most = fmaxf(most, v);
        });
        least = -wave_max(-least);
        most = wave_max(most);
        float *l = (float *)s.part, *h = l + kWaves;
        __syncthreads();
        if (lane == 0) { l[wave] = least; h[wave] = most; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) { least = fminf(least, l[i]); most = fmaxf(most, h[i]); }
        m = s.count;
        __syncthreads();
        lo = least;
        hi = most;
        return m;
    }
    // The pairs of m numbers, dealt to the threads: i with those from .. to - 1.
    struct Pairs {
        int i, from, to;
        __device__ __forceinline__ explicit Pairs(int m)
        {
            const int log = m <= 64 ? 6 : m <= 128 ? 7 : m <= 256 ? 8 : 9;
            const int part = threadIdx.x >> log, share = (m + (kRowThreads >> log) - 1) / (kRowThreads >> log);
            i = threadIdx.x & ((1 << log) - 1);
            from = part * share;
            to = from + share < m ? from + share : m;
        }
    };
    // For each of m logits in `few`: what those before it in the order add up to, and how many they are.
    template <bool MASS>
    __device__ __forceinline__ void compare(int m)
    {
        const Pairs p(m);
        if ((int)threadIdx.x < m) {
            s.few_amount[threadIdx.x] = amount<MASS>(s.few[threadIdx.x]);
            s.few_before[threadIdx.x] = 0;
            s.few_rank[threadIdx.x] = 0;
        }
        __syncthreads();
        if (p.i < m) {
            const float v = s.few[p.i];
            const int at = s.few_at[p.i];
            whole_t before = 0;
            int rank = 0;
#pragma unroll 4
            for (int j = p.from; j < p.to; ++j)
                if (s.few[j] > v || (s.few[j] == v && s.few_at[j] < at)) { before += s.few_amount[j]; ++rank; }
            if (rank) {
                atomicAdd(&s.few_before[p.i], before);
                atomicAdd(&s.few_rank[p.i], rank);
            }
        }
        __syncthreads();
    }
    // The border is the one of m logits in `few` that reaches `want`.
    template <bool MASS>
    __device__ __forceinline__ void border_among(int m, whole_t want)
    {
        compare<MASS>(m);
        // (where rounding leaves all of them short of it: the last one)
        const int i = threadIdx.x;
        if (i < m && s.few_before[i] < want && (s.few_before[i] + s.few_amount[i] >= want || s.few_rank[i] == m - 1)) { s.border = s.few[i]; s.place = s.few_at[i]; }
        __syncthreads();
        border = s.border;
        last = s.place;
        __syncthreads();
    }
    // Among logits lo .. hi, too many to be compared.
    template <bool MASS>
    __device__ __forceinline__ void divide(float lo, float hi, whole_t want)
    {
        while (lo < hi) {
            s.bins[threadIdx.x] = 0;
            __syncthreads();
            const Intervals in(lo, hi);
            sweep(lo, hi, [&](float v, int i) __attribute__((always_inline)) {
                if (inside(v, i)) atomicAdd(&s.bins[in.of(v)], amount<MASS>(v));
            });
            __syncthreads();
            whole_t before;
            const int b = first_to_reach<whole_t>(s.bins[threadIdx.x], want, before);
            want -= before;
            float low = 0.f, high = 0.f;
            const int m = collect(lo, hi, [&](float v, int i) __attribute__((always_inline)) { return in.of(v) == b && inside(v, i); }, low, high);
            if (m <= kSampleFew) {
                border_among<MASS>(m, want);
                return;
            }
            lo = low;
            hi = high;
        }
        // all are equal: so many of them, by index (where rounding asks for more than there are: all)
        const whole_t one = amount<MASS>(lo), some = one ? (want + one - 1) / one : 1;
        const float old = border;
        const int end = last;
        auto equal = [&](float v, int i) __attribute__((always_inline)) { return v == lo && (lo > old || i <= end); };
        for (int i = threadIdx.x; i < a.n_slices; i += kRowThreads) s.more[i] = 0;
        __syncthreads();
        sweep(lo, lo, [&](float v, int i) __attribute__((always_inline)) {
            if (equal(v, i)) atomicAdd(&s.more[i >> a.slice_shift], (whole_t)1);
        });
        __syncthreads();
        whole_t before, all = 0;
        for (int i = 0; i < a.n_slices; ++i) all += s.more[i];
        const whole_t count = some < all ? some : all;
        const int slice = first_to_reach<whole_t>((int)threadIdx.x < a.n_slices ? s.more[threadIdx.x] : 0, count, before);
        border = lo;
        last = place_in(slice, count - before, [&](float v, int i) __attribute__((always_inline)) { return equal(v, i) ? (whole_t)1 : (whole_t)0; });
    }
    // In a slice: the first index at which numbers f(logit, index), added up, reach `want` (at least 1; or all of them, where rounding leaves them short of it).
    template <typename F>
    __device__ __forceinline__ int place_in(int slice, whole_t want, F f)
    {
        const int len = 1 << a.slice_shift;
        whole_t before = 0;
        if (threadIdx.x == 0) s.place = 0;
        for (int c = 0; c < len; c += 4 * kRowThreads) {
            float x[4];
            const int i0 = slice * len + c + 4 * (int)threadIdx.x;
            load4<T>(a, of_row, i0, infinite, x);
            whole_t m[4], mine = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) { m[e] = f(x[e], i0 + e); mine += m[e]; }
            const whole_t upto = wave_scan(mine);
            __syncthreads();
            if (lane == 63) s.whole_part[wave] = upto;
            __syncthreads();
            whole_t now = before + upto - mine;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                if (i < wave) now += s.whole_part[i];
                before += s.whole_part[i];
            }
            // (the last one that is not 0 so far, if it is not reached)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (now < want && m[e] > 0 && (now + m[e] >= want || now + m[e] == before)) s.place = i0 + e;
                now += m[e];
            }
            if (before >= want) break;   // (the same for all)
        }
        __syncthreads();
        const int place = s.place;
        __syncthreads();
        return place;
    }

    __device__ __forceinline__ whole_t least() const
    {
        return rules.min_p > 0.f ? (whole_t)ceil((rules.min_p < 1.f ? (double)rules.min_p : 1.0) * (double)(1ull << a.shift)) : 0;
    }
    // The smallest logit whose weight is not below min_p: 65 parts of an interval at a time, logits as whole numbers in their order.
    __device__ __forceinline__ float smallest_to_weigh(whole_t weight) const
    {
        auto ordered = [](float v) __attribute__((always_inline)) { const uint32_t u = __float_as_uint(v); return (int64_t)(u >> 31 ? ~u : u | 0x80000000u); };
        auto value = [](int64_t o) __attribute__((always_inline)) { return __uint_as_float(o >> 31 & 1 ? (uint32_t)o & 0x7fffffffu : ~(uint32_t)o); };
        int64_t lo = ordered(-INFINITY), hi = ordered((float)scale.top);   // (lo: too little; hi: enough)
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + 64) / 65, mine = lo + step * (lane + 1) < hi ? lo + step * (lane + 1) : hi;
            const whole_t enough = __builtin_amdgcn_ballot_w64(scale.weight(value(mine)) >= weight);
            const int first = enough ? __builtin_ctzll(enough) : 64;   // (the same for all waves)
            const int64_t below = first > 0 ? lo + step * first : lo;
            const int64_t above = first < 64 ? lo + step * (first + 1) : hi;
            lo = below < hi ? below : hi - 1;
            hi = above < hi ? above : hi;
        }
        return value(hi);
    }

    __device__ __forceinline__ void done(int token, float v, double sum) const
    {
        a.token[row] = token;
        if (a.logprob) a.logprob[row] = rules.greedy ? 0.f : (float)(((double)v - scale.top) / (double)rules.temperature - log(sum / (double)(1ull << a.shift)));
    }
    // The first that random number u falls on, of whole sums up to `all`: at least 1, at most all.
    __device__ __forceinline__ double goal(double all) const
    {
        const float u = a.uniform[row];
        return u > 0.f ? (u < 1.f ? (double)u * all : all) : 0.0;   // (a NaN: 0)
    }

    // top_k, where the logits down to the border's interval are few: all that follows among these.
    __device__ __forceinline__ void draw_among(int m)
    {
        compare<true>(m);
        const int i = threadIdx.x;
        const bool mine = i < m;
        const whole_t amount = mine ? s.few_amount[i] : 0, before = mine ? s.few_before[i] : 0;
        const bool k = mine && s.few_rank[i] < rules.top_k;
        __syncthreads();
        if (threadIdx.x == 0) { s.total = 0; s.whole_before = 0; }
        __syncthreads();
        if (k) atomicAdd(&s.total, amount);
        __syncthreads();
        const whole_t all = s.total;
        whole_t want = all;
        if (rules.top_p < 1.f && !rules.greedy) {
            const double p = rules.top_p > 0.f ? ceil((double)rules.top_p * (double)all) : 0.0;
            want = p >= (double)all ? all : (whole_t)p;
            if (want < 1) want = 1;
        }
        const bool kept = k && amount > 0 && before < want && (rules.greedy || amount >= least());
        if (mine) {
            s.few_before[i] = kept ? amount : 0;
            s.few_below[i] = 0;
        }
        if (kept) atomicAdd(&s.whole_before, amount);
        __syncthreads();
        const whole_t sum = s.whole_before;
        const double g = goal((double)sum);
        whole_t to = (whole_t)g + 1;
        if (to > sum) to = sum;
        const Pairs p(m);
        if (p.i < m) {
            const int at = s.few_at[p.i];
            whole_t below = 0;
#pragma unroll 4
            for (int j = p.from; j < p.to; ++j)
                if (s.few_at[j] < at) below += s.few_before[j];
            if (below) atomicAdd(&s.few_below[p.i], below);
        }
        __syncthreads();
        if (kept && s.few_below[i] < to && s.few_below[i] + amount >= to) done(s.few_at[i], s.few[i], (double)sum);
    }

    __device__ __forceinline__ void draw()
    {
        // ---- the slices meet
        const int n = a.n_slices;
        for (int i = threadIdx.x; i < n; i += kRowThreads) {
            const float most = slices[i].most;
            const bool none = most == -INFINITY || (infinite && most < INFINITY);
            const float own = infinite ? 0.f : most;
            s.factor[i] = none ? 0.0 : exp2(((double)own - scale.top) * scale.per);
            s.later[i] = none ? kSampleBins : (int)fminf(scale.first - scale.interval(own), (float)kSampleBins);
        }
        __syncthreads();
        const bool counted = rules.top_k > 0;
        // (the last interval is what lies behind all others, in whichever slice: not added up)
        double mine = 0.0, all = 0.0;
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const int j = (int)threadIdx.x - s.later[i];
            const double f = s.factor[i], v = (double)slices[i].bins[j >= 0 ? j : 0];
            mine += j >= 0 ? (counted ? v : f * v) : 0.0;
            all += f > 0.0 || (counted && !infinite && slices[i].most > -INFINITY) ? (counted ? 1.0 : f) * (double)slices[i].all : 0.0;
        }
        if (threadIdx.x == kSampleBins - 1) mine = 0.0;
        const whole_t low = least();
        bool by_bins = false, listed = false;   // whether the slices' kept weights come from their histograms; whether `few` holds the border's interval
        int edge = kSampleBins, m = 0;          // the border's interval
        if (counted) {
            const double k = (double)rules.top_k < all ? (double)rules.top_k : all;
            double before;
            const int b = first_to_reach<double>(mine, k, before);
            const Interval in(scale, b);
            float lo = 0.f, hi = 0.f;
            m = collect(in.low, INFINITY, [&](float v, int) __attribute__((always_inline)) { return scale.bin(v) <= b; }, lo, hi);
            if (m <= kSampleFew) {
                draw_among(m);
                return;
            }
            if ((double)rules.top_k < all) {
                const int upto = collect(in.low, in.high, [&](float v, int) __attribute__((always_inline)) { return scale.bin(v) == b; }, lo, hi);
                if (upto <= kSampleFew) border_among<false>(upto, (whole_t)(k - before));
                else divide<false>(lo, hi, (whole_t)(k - before));
            }
            if (rules.top_p < 1.f && !rules.greedy) {
                // (their weights' sum first)
                const whole_t sum = sum_kept();
                const double p = rules.top_p > 0.f ? ceil((double)rules.top_p * (double)sum) : 0.0;
                whole_t want = p >= (double)sum ? sum : (whole_t)p;
                if (want < 1) want = 1;
                m = collect(border, INFINITY, [&](float v, int i) __attribute__((always_inline)) { return inside(v, i); }, lo, hi);
                if (m <= kSampleFew) border_among<true>(m, want);
                else divide<true>(lo, hi, want);
            }
        } else {
            by_bins = true;
            // (of two borders the higher one counts; min_p's is known by itself, so that one interval at most is collected)
            int p_edge = kSampleBins;
            double want = 0.0, before = 0.0;
            if (rules.top_p < 1.f) {
                want = rules.top_p > 0.f ? (double)rules.top_p * all : 0.0;
                if (!(want >= 1.0)) want = 1.0;
                p_edge = first_to_reach<double>(mine, want, before);
            }
            const float smallest = low > 0 ? smallest_to_weigh(low) : -INFINITY;
            edge = low > 0 && scale.bin(smallest) < p_edge ? scale.bin(smallest) : p_edge;
            if (edge < kSampleBins) {
                const Interval in(scale, edge);
                float lo = 0.f, hi = 0.f;
                m = collect(in.low, in.high, [&](float v, int) __attribute__((always_inline)) { return scale.bin(v) == edge; }, lo, hi);
                listed = m <= kSampleFew;
                if (edge == p_edge) {
                    const double rest = ceil(want - before);
                    const whole_t left = rest > 1.0 ? (whole_t)rest : 1;
                    if (listed) border_among<true>(m, left);
                    else divide<true>(lo, hi, left);
                }
                if (border < smallest) { border = smallest; last = 0x7fffffff; }
            }
        }
        if (counted && low > 0 && scale.weight(border) < low) {
            border = smallest_to_weigh(low);
            last = 0x7fffffff;
        }
        // ---- the kept weights of every slice: whole intervals, and what is kept of the border's
        for (int i = threadIdx.x; i < n; i += kRowThreads) s.more[i] = 0;
        __syncthreads();
        if (by_bins && listed) {
            if ((int)threadIdx.x < m && inside(s.few[threadIdx.x], s.few_at[threadIdx.x])) atomicAdd(&s.more[s.few_at[threadIdx.x] >> a.slice_shift], scale.weight(s.few[threadIdx.x]));
        } else if (!by_bins || edge < kSampleBins) {
            sweep(border, by_bins ? Interval(scale, edge).high : INFINITY, [&](float v, int i) __attribute__((always_inline)) {
                if (inside(v, i) && (!by_bins || scale.bin(v) == edge)) atomicAdd(&s.more[i >> a.slice_shift], scale.weight(v));
            });
        }
        __syncthreads();
        for (int i = wave; i < n; i += kWaves) {
            whole_t sum = 0;
            if (by_bins && s.factor[i] > 0.0) {
                if (edge == kSampleBins) sum = lane == 63 ? slices[i].all : 0;
                else {
#pragma unroll 4
                    for (int j = lane; j < edge - s.later[i]; j += 64) sum += slices[i].bins[j];
                }
                sum = wave_scan(sum);
            }
            if (lane == 63) {
                const double k = (double)sum * s.factor[i] + (double)s.more[i];
                s.kept[i] = k < (double)(1 << a.slice_shift) / 2 ? 0.0 : k;   // (all of its weights might be rounded to 0)
            }
        }
        __syncthreads();
        // ---- the draw: a slice, then its token
        static_assert(kMaxSlices == 64, "a slice for each lane");
        const double of = lane < n ? s.kept[lane] : 0.0, upto = wave_scan(of);
        const double sum = __longlong_as_double(((long long)__builtin_amdgcn_readlane((int)(__double_as_longlong(upto) >> 32), 63) << 32) |
                                                (uint32_t)__builtin_amdgcn_readlane((int)__double_as_longlong(upto), 63));
        const double to = goal(sum);
        // (one that has any: the first whose sum with those before it is above the goal, or the last)
        const whole_t some = __builtin_amdgcn_ballot_w64(of > 0.0), above = __builtin_amdgcn_ballot_w64(of > 0.0 && upto > to);
        const int slice = above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some | 1);
        const double start = upto - of;
        const double before = __longlong_as_double(((long long)__builtin_amdgcn_readlane((int)(__double_as_longlong(start) >> 32), slice) << 32) |
                                                   (uint32_t)__builtin_amdgcn_readlane((int)__double_as_longlong(start), slice));
        const double rest = to - before;
        const whole_t want = rest > 0.0 ? (whole_t)rest + 1 : 1;
        const int place = place_in(slice, want, [&](float v, int i) __attribute__((always_inline)) {
            const whole_t w = inside(v, i) ? scale.weight(v) : 0;
            return w;
        });
        if (threadIdx.x == 0) done(place, as_logit(load_f32(of_row, (size_t)place), infinite), sum);
    }
    __device__ __forceinline__ whole_t sum_kept()
    {
        whole_t mine = 0;
        sweep(border, INFINITY, [&](float v, int i) __attribute__((always_inline)) { if (inside(v, i)) mine += scale.weight(v); });
        const whole_t upto = wave_scan(mine);
        if (lane == 63) s.whole_part[wave] = upto;
        __syncthreads();
        whole_t all = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) all += s.whole_part[i];
        __syncthreads();
        return all;
    }
};

// FUSED: the block looks at its row's slices itself.  grid: rows
template <typename T, bool FUSED>
__global__ __launch_bounds__(kRowThreads) void sample_rows_kernel(const SampleArgs a)
{
    __shared__ RowShared shared;
    const int row = blockIdx.x;
    const RowRules rules(a, row);
    const Slice *slices = a.slices + (size_t)row * a.n_slices;
    if constexpr (FUSED) {
        __shared__ SliceShared<kRowThreads> look;
        __shared__ Slice own[kFusedSlices];
        for (int i = 0; i < a.n_slices; ++i) look_at_slice<T, kRowThreads, 1>(a, rules, (const T *)a.logits + (size_t)row * a.ld, i, look, own + i);
        slices = own;
    }
    float most = -INFINITY;
    for (int i = threadIdx.x & 63; i < a.n_slices; i += 64) most = fmaxf(most, slices[i].most);
    most = wave_max(most);
    if (most == -INFINITY) {   // no token
        if (threadIdx.x == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = __uint_as_float(0x7fc00000u);
        }
        return;
    }
    RowSampler<T> sampler(a, shared, slices, rules, row, most);
    sampler.draw();
}

}  // namespace anpd
