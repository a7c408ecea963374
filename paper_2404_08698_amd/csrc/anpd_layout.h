// Storage types, and where a cached key or value lies in the pool: shared by the verification step and by the operators on caches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace anpd {

typedef uint16_t bf16_t;  // bfloat16 storage
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

__device__ __forceinline__ float bf16_to_f32(bf16_t b) { return __uint_as_float((uint32_t)b << 16); }

// round to nearest, ties to even (finite inputs)
__device__ __forceinline__ bf16_t f32_to_bf16(float f)
{
    uint32_t u = __float_as_uint(f);
    u += 0x7fffu + ((u >> 16) & 1u);
    return (bf16_t)(u >> 16);
}

__device__ __forceinline__ float load_f32(const float *p, size_t i) { return p[i]; }
__device__ __forceinline__ float load_f32(const bf16_t *p, size_t i) { return bf16_to_f32(p[i]); }
__device__ __forceinline__ void store_kv(float *p, size_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store_kv(bf16_t *p, size_t i, float v) { p[i] = f32_to_bf16(v); }

// two floats rounded to bf16 (nearest even) side by side, one instruction
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, b16x2));
}

// Page layout of the generic path: [page][layer][k|v][head][token in page][head_dim].
__device__ __forceinline__ size_t kv_offset(int page, int layer, int n_layers, int kv, int head, int n_heads,
                                            int tok_in_page, int page_tokens, int head_dim)
{
    return ((((size_t)page * n_layers + layer) * 2 + kv) * n_heads + head) * ((size_t)page_tokens * head_dim) +
           (size_t)tok_in_page * head_dim;
}

// ------------------------------------------------------ fast-path KV cache
//
// The fast path keeps K and V in MFMA-fragment order inside each (page, layer,
// k|v, head) block of 16 tokens x head_dim (page_tokens is 16 on this path):
//   K: [dim / 32][lane = 16 * ((dim % 32) / 8) + token][dim % 8]     A operand of 16x16x32 (rows = keys)
//   V: [dim / 16][lane = 16 * (token / 4) + dim % 16][token % 4]     A operand of 16x16x16 (rows = dims)
// so a wave loads a page's K (and V) tile with fully coalesced reads.
__host__ __device__ __forceinline__ size_t kvf_base(int page, int layer, int n_layers, int kv, int head, int n_heads,
                                                    int head_dim)
{
    return ((((size_t)page * n_layers + layer) * 2 + kv) * n_heads + head) * ((size_t)16 * head_dim);
}
__host__ __device__ __forceinline__ size_t kf_elem(int tok, int dim)
{
    return ((size_t)(dim >> 5) * 64 + (size_t)((dim >> 3) & 3) * 16 + tok) * 8 + (dim & 7);
}
__host__ __device__ __forceinline__ size_t vf_elem(int tok, int dim)
{
    return ((size_t)(dim >> 4) * 64 + (size_t)(tok >> 2) * 16 + (dim & 15)) * 4 + (tok & 3);
}

}  // namespace anpd
