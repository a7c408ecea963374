// Drawing tokens from logits: host half.  The kernels and their reasons are in anpd_sample.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "anpd_cache.h"
#include "anpd_sample.h"

using namespace anpd;

namespace {

constexpr int kGroup = 256;   // rows of a launch, whose slices the workspace holds

template <bool FUSED>
void launch_rows(const SampleArgs &a, unsigned rows, hipStream_t st)
{
    if (a.f32) hipLaunchKernelGGL((sample_rows_kernel<float, FUSED>), dim3(rows), dim3(kRowThreads), 0, st, a);
    else hipLaunchKernelGGL((sample_rows_kernel<bf16_t, FUSED>), dim3(rows), dim3(kRowThreads), 0, st, a);
}
template <int THREADS>
void launch_slices(const SampleArgs &a, unsigned rows, hipStream_t st)
{
    const dim3 grid((unsigned)a.n_slices, rows);
    if (a.f32) hipLaunchKernelGGL((sample_slices_kernel<float, THREADS>), grid, dim3(THREADS), 0, st, a);
    else hipLaunchKernelGGL((sample_slices_kernel<bf16_t, THREADS>), grid, dim3(THREADS), 0, st, a);
}

int slices_of(int32_t vocab) { return ((vocab - 1) >> slice_shift(vocab)) + 1; }

}  // namespace

extern "C" {

size_t anpd_sample_workspace_bytes(int32_t rows, int32_t vocab)
{
    if (rows < 0 || vocab < 1 || vocab > kSampleMaxVocab) {
        fail(ANPD_E_INVAL, "anpd_sample_workspace_bytes: rows must be >= 0, vocab in 1..%d", kSampleMaxVocab);
        return 0;
    }
    const int n = slices_of(vocab);
    return n <= kFusedSlices ? 0 : align_up((size_t)(rows < kGroup ? rows : kGroup) * n * sizeof(Slice));
}

int32_t anpd_sample(const void *logits, int64_t ld, int32_t dtype, int32_t rows, int32_t vocab, const anpd_sample_rules *rules, const float *uniform,
                    int32_t *out_token, float *out_logprob, void *workspace, size_t workspace_bytes, void *stream)
{
    const char *who = "anpd_sample";
    if (dtype != ANPD_F32 && dtype != ANPD_BF16) return fail(ANPD_E_INVAL, "%s: unknown dtype", who);
    if (rows < 0) return fail(ANPD_E_INVAL, "%s: %d rows", who, rows);
    if (vocab < 1 || vocab > kSampleMaxVocab) return fail(ANPD_E_INVAL, "%s: vocab must be in 1..%d", who, kSampleMaxVocab);
    if (ld < vocab) return fail(ANPD_E_INVAL, "%s: rows are %d elements wide and %lld apart", who, vocab, (long long)ld);
    SampleArgs a;
    std::memset(&a, 0, sizeof(a));
    a.temperature = a.top_p = 1.f;
    if (rules) {
        if (!(rules->temperature >= 0.f) || std::isinf(rules->temperature)) return fail(ANPD_E_INVAL, "%s: temperature must be finite and >= 0", who);
        if (rules->top_k < 0) return fail(ANPD_E_INVAL, "%s: top_k must be >= 0", who);
        if (!(rules->top_p >= 0.f && rules->top_p <= 1.f) || !(rules->min_p >= 0.f && rules->min_p <= 1.f)) return fail(ANPD_E_INVAL, "%s: top_p and min_p must be in 0..1", who);
        a.temperature = rules->temperature;
        a.top_k = rules->top_k;
        a.top_p = rules->top_p;
        a.min_p = rules->min_p;
        a.temperatures = rules->temperatures;
        a.top_ks = rules->top_ks;
        a.top_ps = rules->top_ps;
        a.min_ps = rules->min_ps;
        if ((((uintptr_t)a.temperatures | (uintptr_t)a.top_ks | (uintptr_t)a.top_ps | (uintptr_t)a.min_ps) & 3) != 0)
            return fail(ANPD_E_INVAL, "%s: an array of the rules is not aligned to its type", who);
    }
    if (rows == 0) return ANPD_OK;
    if (!logits || !uniform || !out_token) return fail(ANPD_E_INVAL, "%s: NULL argument", who);
    if ((((uintptr_t)uniform | (uintptr_t)out_token | (uintptr_t)out_logprob) & 3) != 0 || ((uintptr_t)logits & (dtype == ANPD_F32 ? 3 : 1)) != 0)
        return fail(ANPD_E_INVAL, "%s: an argument is not aligned to its type", who);
    a.logits = logits;
    a.ld = ld;
    a.uniform = uniform;
    a.token = out_token;
    a.logprob = out_logprob;
    a.vocab = vocab;
    a.f32 = dtype == ANPD_F32;
    a.wide = ((uintptr_t)logits & (a.f32 ? 15 : 7)) == 0 && ld % 4 == 0;
    a.n_slices = slices_of(vocab);
    a.slice_shift = slice_shift(vocab);
    // (a row's weights add up to 2^62 at most)
    a.shift = 51;
    while ((1ull << (62 - a.shift)) < (uint64_t)vocab) --a.shift;
    const size_t need = anpd_sample_workspace_bytes(rows, vocab);
    if (need > 0) {
        if (!workspace || ((uintptr_t)workspace & 255) != 0) return fail(ANPD_E_INVAL, "%s: workspace must be a 256-byte aligned device buffer", who);
        if (workspace_bytes < need) return fail(ANPD_E_CAPACITY, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
    }
    OnDevice on;
    int32_t rc = on.enter_of(who, logits);
    if (rc != ANPD_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    a.slices = (Slice *)workspace;
    // (a launch has fewer than 2^32 threads)
    const int64_t group = need > 0 ? kGroup : 1 << 21;
    for (int64_t row = 0; row < rows; row += group) {
        const unsigned n = (unsigned)(rows - row < group ? rows - row : group);
        SampleArgs g = a;
        g.logits = (const char *)logits + (size_t)row * ld * (a.f32 ? 4 : 2);
        g.uniform += row;
        g.token += row;
        if (g.logprob) g.logprob += row;
        if (g.temperatures) g.temperatures += row;
        if (g.top_ks) g.top_ks += row;
        if (g.top_ps) g.top_ps += row;
        if (g.min_ps) g.min_ps += row;
        if (need == 0) launch_rows<true>(g, n, st);
        else {
            if (a.slice_shift == 12) launch_slices<256>(g, n, st);
            else launch_slices<1024>(g, n, st);
            HIP_TRY(hipGetLastError());
            launch_rows<false>(g, n, st);
        }
        HIP_TRY(hipGetLastError());
    }
    return ANPD_OK;
}

}  // extern "C"
