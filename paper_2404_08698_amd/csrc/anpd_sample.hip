// Drawing tokens from logits: host half.  The kernels and their reasons are in anpd_sample.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "anpd_cache.h"
#include "anpd_sample.h"

using namespace anpd;

extern "C" {

int32_t anpd_sample(const void *logits, int64_t ld, int32_t dtype, int32_t rows, int32_t vocab, const anpd_sample_rules *rules, const float *uniform,
                    int32_t *out_token, float *out_logprob, void *stream)
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
    a.rows = rows;
    a.vocab = vocab;
    a.f32 = dtype == ANPD_F32;
    a.wide = ((uintptr_t)logits & (a.f32 ? 15 : 7)) == 0 && ld % 4 == 0;
    // (all weights of a row fit in 63 bits)
    a.shift = 51;
    while (((uint64_t)vocab << a.shift) > (1ull << 62)) --a.shift;
    OnDevice on;
    int32_t rc = on.enter_of(who, logits);
    if (rc != ANPD_OK) return rc;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)rows);
    if (vocab <= 256 * kSampleHeld) hipLaunchKernelGGL((sample_kernel<256, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((sample_kernel<1024, false>), grid, dim3(1024), 0, st, a);
    HIP_TRY(hipGetLastError());
    return ANPD_OK;
}

}  // extern "C"
