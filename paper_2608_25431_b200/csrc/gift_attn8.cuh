// Attention over 8-bit pages: what its kernels share.
#pragma once
#include "gift_attn.cuh"
#include "gift_kv8.cuh"
#include "gift_tc.cuh"

namespace gift {

struct Attn8Args : AttnArgs {
    uint32_t codes;                  // bytes of K's (or V's) codes of one token; V's, then the scales, lie behind
    float cap_in, cap_out;           // scale / softcap, softcap * log2(e); cap_out 0: no cap
    const float* slopes;
    uint32_t half;                   // q and out are fp16, not bf16
    uint32_t head_ways;              // few rows: K/V heads that a CTA's warps share out (kv_heads counts groups of them)
    uint32_t copy_run;               // many rows: tokens that are one copy, the largest power of two up to a tile that divides the page
    uint32_t whole_steps;            // few rows: a page is whole steps of a warp
};

constexpr float LOG2_E = 1.4426950408889634f;
constexpr uint32_t FOUND_NAN = 1u << 31;  // beside a piece's status bits: codes of NaN in V became 0
constexpr float NOTHING = -3e38f;        // the maximum before anything is seen: finite, so that no difference with it is NaN

__device__ __forceinline__ float fast_rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// tanh times cap, by two forms.  Up to 0.75: tanh(u) / u as a polynomial of u^2, fitted for the least relative error (3.7e-8 as stored;
// 2^-22.4 with the roundings).  Above: 1 - 2 / (e^2u + 1), whose error is 2^-21 at most (of the exponential 2^-22 and of the reciprocal 2^-23, both
// relative).  A number's form depends on itself alone, and so does its value: not on what else is in its step.
constexpr float TANH_NEAR = 0.75f;
__device__ __forceinline__ float tanh_c(int i)
{
    constexpr float C[5] = {-4.769490100e-3f, 1.966491342e-2f, -5.339025706e-2f, 1.332652122e-1f, -3.333306909e-1f};
    return C[i];
}
// Two numbers below the border: steps all of whose numbers are (for a cap of 30, scores up to 22) take this, without exponential and reciprocal.
__device__ __forceinline__ uint64_t capped_near(uint64_t u, uint64_t cap2)
{
    const uint64_t x = mul2(u, u);
    uint64_t p = pair2(tanh_c(0), tanh_c(0));
#pragma unroll
    for (int i = 1; i < 5; i++) p = fma2(p, x, pair2(tanh_c(i), tanh_c(i)));
    return mul2(mul2(u, cap2), fma2(p, x, pair2(1.f, 1.f)));
}
// Any number; below the border to the same bit.
__device__ __forceinline__ float capped(float u, float cap)
{
    const float x = u * u;
    float p = tanh_c(0);
#pragma unroll
    for (int i = 1; i < 5; i++) p = fmaf(p, x, tanh_c(i));
    const float near = __fmul_rn(__fmul_rn(u, cap), fmaf(p, x, 1.f)), far = cap * (1.f - 2.f * fast_rcp(fast_exp2(u * (2.f * LOG2_E)) + 1.f));
    return fabsf(u) <= TANH_NEAR ? near : far;
}

// Power-of-two factors, made of exponents: a value with exponent field e, or 9 where that is less, becomes one of about
// 2^8: in fp16 well above what it rounds (2^-14), with room for one that is 2^7 larger.  e = 255: infinities and NaN stay.
__device__ __forceinline__ uint32_t top_exponent(uint32_t magnitude) { return magnitude >> 23 < 9u ? 9u : magnitude >> 23; }
__device__ __forceinline__ float to_half_range(uint32_t e) { return e == 255u ? 1.f : __uint_as_float((262u - e) << 23); }
__device__ __forceinline__ float from_half_range(uint32_t e) { return e == 255u ? 1.f : __uint_as_float((e - 8u) << 23); }
// The reciprocal of a power of two, exact.
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float(0x7F000000u - __float_as_uint(x)); }
// The largest value that fits fp16 by e's factor.
__device__ __forceinline__ float half_range_end(uint32_t e) { return __uint_as_float((e > 247u ? 254u : e + 7u) << 23); }

// Which of the 64 tokens from t0 a row sees where a window ends among them, as bits: those from position x - window + 1 on.
__device__ __forceinline__ uint64_t in_window64(uint32_t window, uint32_t x, uint32_t t0)
{
    const uint32_t low = x >= window ? x - window + 1u : 0u;
    if (low <= t0) return ~0ull;
    return low - t0 >= 64u ? 0ull : ~0ull << (low - t0);
}

template <class T> __device__ __forceinline__ T not_a_number();
template <> __device__ __forceinline__ float not_a_number<float>() { return __uint_as_float(0x7FC00000u); }
template <> __device__ __forceinline__ uint16_t not_a_number<uint16_t>() { return 0x7FFFu; }             // bf16 and fp16 alike

// Whether a word of four codes holds one that is NaN.
__device__ __forceinline__ bool codes_nan(uint32_t w) { return (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0u; }
// The word with those codes 0.
__device__ __forceinline__ uint32_t codes_without_nan(uint32_t w)
{
    const uint32_t bad = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;      // one bit a byte
    return w & ~((bad >> 7) * 255u);
}

// Where tokens may be hidden from some row, codes of NaN in V enter the products as 0.  This gives the rows that see them their NaN, in the
// columns that have it, when the products are done: `tokens` (32 at most) from t0 of request r, K/V head h, are read again from the pages.  A
// warp's, each lane with a row of its own (`there`: it has one): the request's i-th, `row` of the step, whose results lie at `to`.
template <int D, class T>
static __device__ __noinline__ void put_nan(const Attn8Args& a, uint32_t r, uint32_t h, uint32_t have, uint32_t want, uint32_t row, uint32_t i,
                                            uint32_t t0, uint32_t tokens, bool there, T* to)
{
    const uint32_t lane = threadIdx.x & 31u, t = t0 + lane;
    const char* codes = a.pages + a.codes + (uint64_t)h * D;
    bool odd = false;
    if (lane < tokens && t < want) {
        const uint32_t b = a.b.page.quot(t), page = (uint32_t)a.b.table[(uint64_t)r * a.b.max_blocks + b];
        if (page < a.b.n_pages) {
            codes += ((uint64_t)page * a.b.page_tokens + (t - b * a.b.page_tokens)) * a.token_bytes;
#pragma unroll 1
            for (uint32_t c = 0; c < (uint32_t)D; c += 4) odd |= codes_nan(*reinterpret_cast<const uint32_t*>(codes + c));
        }
    }
    uint32_t found = __ballot_sync(0xFFFFFFFFu, odd);
    if (found == 0u) return;
    uint32_t sees = there ? (uint32_t)row_sees64(a, have, want, row, i, t0) : 0u;
    if (a.window) sees &= (uint32_t)in_window64(a.window, have + i, t0);
#pragma unroll 1
    for (; found; found &= found - 1u) {
        const uint32_t k = __ffs(found) - 1;
        const char* p = reinterpret_cast<const char*>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)codes, k));
        if (sees >> k & 1u)
#pragma unroll 1
            for (uint32_t c = 0; c < (uint32_t)D; c++)
                if ((p[c] & 0x7F) == 0x7F) to[c] = not_a_number<T>();
    }
}

__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, uint32_t bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ float2 lds_pair(uint32_t at)
{
    float2 x;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at) : "memory");
    return x;
}
// Four codes as two pairs.
__device__ __forceinline__ void four_codes(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    asm("{\n .reg .b16 x, y;\n mov.b32 {x, y}, %2;\n cvt.rn.f16x2.e4m3x2 %0, x;\n cvt.rn.f16x2.e4m3x2 %1, y;\n}" : "=r"(lo), "=r"(hi) : "r"(w));
}

// Two results as a pair of q's type.
__device__ __forceinline__ uint32_t pack_out(const Attn8Args& a, float lo, float hi)
{
    return a.half ? pack2<__half>(lo, hi) : pack2<__nv_bfloat16>(lo, hi);
}

}  // namespace gift
