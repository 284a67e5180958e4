// The 8-bit pool: layout of a token, host checks, e4m3 codes.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gift_kv.cuh"

namespace gift {

// Host checks of a pool of 16 or 8 bits.
inline int any_pool_args_ok(const gift_kv_pool* p)
{
    if (!p) return GIFT_E_INVAL;
    if (p->dtype != GIFT_E4M3) return pool_args_ok(p);
    gift_kv_pool as16 = *p;
    as16.dtype = GIFT_BF16;
    const int rc = pool_args_ok(&as16);
    if (rc != GIFT_OK) return rc;
    return p->head_dim % 16 ? GIFT_E_ALIGN : GIFT_OK;
}

// A token of an 8-bit pool: K codes, V codes, scales.
struct Kv8 {
    uint64_t token;                  // bytes
    uint32_t codes;                  // of K, or of V: heads * head_dim bytes
};
inline Kv8 kv8_layout(const gift_kv_pool* p)
{
    Kv8 k;
    k.token = GIFT_KV8_TOKEN_BYTES(p->n_heads, p->head_dim);
    k.codes = p->n_heads * p->head_dim;
    return k;
}

// Two e4m3 codes as a pair of fp16 numbers, exact.
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t two)
{
    uint32_t r;
    asm("{\n .reg .b16 c;\n cvt.u16.u32 c, %1;\n cvt.rn.f16x2.e4m3x2 %0, c;\n}" : "=r"(r) : "r"(two));
    return r;
}
// The codes nearest to lo and hi, in the low 16 bits.
__device__ __forceinline__ uint32_t floats_to_codes(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace gift
