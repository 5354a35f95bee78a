// The KV cache held in 8 bits: layout, number format and device tables, shared by the kernels that build, fill, read
// and attend over it.
//
// Pool: [num_pages, kv_heads, 2 (K, V), 16, head_dim] e4m3 codes; scales: [num_pages, kv_heads, 2] fp32; a stored
// value is code * scale.  The scale of a (page, kv head, K or V) is the smallest power of two s >= 2^-126 with
// amax <= 448 s over the page's finite values.  With powers of two the division by s and the later product with it are
// exact, so the only rounding is the one to 4 significant bits, and a page whose scale has to grow is re-rounded by an
// exponent shift that changes nothing above e4m3's subnormals; a free scale would gain at most one bit of range (not
// of precision: the codes are floating point) and round every earlier code again.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "cpa_device.cuh"
#include "cpa_internal.h"

namespace {

constexpr int kPage = 16;                     // tokens per page

// ---------------------------------------------------------------- tables
// Device tables, int32 words: a header (word 0: what append and decode launches record, 1 tokens, 2 pages, from word
// kBuildWords on what each CTA of the build has found), then cu_seqlens, page_indptr, the page list, the slot map and
// the merge tickets of the decode (zero between launches), each 16-byte aligned.
constexpr int kBuildWords = 4, kBuildCtas = 296, kHeaderWords = 300;   // 300: a multiple of 4
struct q8_tables {
    int32_t* header;
    int32_t* cu_seqlens;     // [B+1]
    int32_t* page_indptr;    // [B+1]
    int32_t* page_indices;   // [page_capacity]
    int32_t* slot_mapping;   // [token_capacity]
    int32_t* tickets;        // [B * Hkv]
};
struct q8_offsets { int64_t cu, indptr, pages, slots, tickets, words; };

inline q8_offsets q8_layout(const cpa_config& c, const cpa_table_dims& d) {
    auto up = [](int64_t w) { return (w + 3) / 4 * 4; };
    q8_offsets o;
    o.cu = kHeaderWords;
    o.indptr = o.cu + up((int64_t)d.num_blocks + 1);
    o.pages = o.indptr + up((int64_t)d.num_blocks + 1);
    o.slots = o.pages + up(d.page_capacity);
    o.tickets = o.slots + up(d.token_capacity);
    o.words = o.tickets + up((int64_t)d.num_blocks * c.num_kv_heads);
    return o;
}
inline q8_tables q8_view(const cpa_config& c, const cpa_table_dims& d, const void* base) {
    const q8_offsets o = q8_layout(c, d);
    int32_t* p = static_cast<int32_t*>(const_cast<void*>(base));
    return {p, p + o.cu, p + o.indptr, p + o.pages, p + o.slots, p + o.tickets};
}

constexpr int32_t kMaxTableBlocks = 1 << 20;

// CPA_OK, or why this configuration or these sizes are refused.
inline int q8_check(const cpa_config* c, const cpa_table_dims* d) {
    if (!c || !d) return CPA_EINVAL;
    if (c->num_q_heads < 1 || c->num_kv_heads < 1 || c->num_q_heads % c->num_kv_heads != 0 || c->num_sms < 0 ||
        !(c->scale > 0.f))
        return CPA_EINVAL;
    if ((c->head_dim != 64 && c->head_dim != 128) || c->page_size != kPage || c->num_q_heads / c->num_kv_heads > 8 ||
        c->num_sms > kMaxPlanSms || c->num_kv_heads > 1024)
        return CPA_EUNSUPPORTED;
    if (d->num_blocks < 1 || d->max_new_tokens < 0 || d->num_pages < 1 || d->page_capacity < 0 || d->token_capacity < 0)
        return CPA_EINVAL;
    // slots are int32, and the pool's rows of 128 bytes are addressed with 32-bit coordinates
    if (d->num_blocks > kMaxTableBlocks || d->page_capacity > (1 << 30) || (int64_t)d->num_pages * kPage > INT32_MAX ||
        (int64_t)d->num_pages * c->num_kv_heads * 32 > INT32_MAX ||
        (int64_t)d->num_blocks * c->num_kv_heads > INT32_MAX)
        return CPA_EUNSUPPORTED;
    return CPA_OK;
}

// Loads of what an earlier launch of the stream may have written.  A programmatic launch begins before that launch has
// ended, so its kernel may use neither non-coherent loads (their data would have to be constant from the kernel's begin)
// nor ordinary ones of a __restrict__ const argument (which the compiler may turn into those, or move in front of the
// wait).  Volatile assembly stays behind the wait, which is volatile assembly too.
__device__ __forceinline__ int32_t ld_i32(const int32_t* p) {
    int32_t v;
    asm volatile("ld.global.s32 %0, [%1];\n" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float ld_f32(const float* p) {
    float v;
    asm volatile("ld.global.f32 %0, [%1];\n" : "=f"(v) : "l"(p));
    return v;
}

// A programmatic launch: the grid may be made ready while the stream's earlier work ends; the kernel waits for that
// work (griddepcontrol.wait) before it reads anything.
template <class... P, class... A>
int q8_launch(void (*kernel)(P...), int grid, int threads, cudaStream_t st, A... args) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)grid);
    lc.blockDim = dim3((unsigned)threads);
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    if (cudaLaunchKernelEx(&lc, kernel, static_cast<P>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return CPA_ECUDA;
    }
    return CPA_OK;
}

// ---------------------------------------------------------------- number format
// Scale of a page whose largest finite magnitude has the fp32 bits `amax`: 448 = 1.75 * 2^8, so the exponent is that of
// amax less 8, and one more when amax's significand is above 1.75.
__device__ __forceinline__ float q8_scale(uint32_t amax) {
    const int e = max((int)((amax + 0x1FFFFFu) >> 23) - 8, 1);      // biased; 1 = 2^-126
    return __uint_as_float((uint32_t)e << 23);
}
// 1 / s of a power of two between 2^-126 and 2^120 (exact)
__device__ __forceinline__ float q8_inverse(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// |x| as fp32 bits for the page's amax; infinities and NaN do not count
__device__ __forceinline__ uint32_t q8_finite_abs(uint32_t bits) {
    const uint32_t a = bits & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0u;
}
// product and quotient that keep subnormals (the file's other arithmetic may flush them)
__device__ __forceinline__ float mul_keep(float a, float b) {
    float d;
    asm("mul.rn.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float div_keep(float a, float b) {
    float d;
    asm("div.rn.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// two values to e4m3, nearest even; beyond 448 (infinities alone get there) to 448; NaN stays NaN
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint16_t v) {
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(d) : "h"(v));
    return d;
}
__device__ __forceinline__ float2 e4m3x2_to_f32(uint16_t v) {
    const uint32_t h = e4m3x2_to_f16x2(v);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// four codes times a factor, to four codes (the re-rounding of a page whose scale grows)
__device__ __forceinline__ uint32_t q8_rescale4(uint32_t codes, float f) {
    const float2 a = e4m3x2_to_f32((uint16_t)codes), b = e4m3x2_to_f32((uint16_t)(codes >> 16));
    return to_e4m3x2(mul_keep(a.x, f), mul_keep(a.y, f)) | (to_e4m3x2(mul_keep(b.x, f), mul_keep(b.y, f)) << 16);
}
// Whether a scale is one that the append calls give (another writer of the pool may have left any).
__device__ __forceinline__ bool q8_power_of_two(float s) { return (__float_as_uint(s) & 0x807FFFFFu) == 0 && s <= 0x1p120f; }
// x / s, by the exact product where s is a power of two
__device__ __forceinline__ float q8_divide(float x, float s, bool power_of_two) {
    return power_of_two ? mul_keep(x, q8_inverse(s)) : div_keep(x, s);
}
// eight bf16 values divided by the scale, to eight codes
__device__ __forceinline__ uint2 q8_codes8(uint4 v, float s) {
    auto two = [&](uint32_t w) {
        return to_e4m3x2(div_keep(__uint_as_float(w << 16), s), div_keep(__uint_as_float(w & 0xFFFF0000u), s));
    };
    return make_uint2(two(v.x) | (two(v.y) << 16), two(v.z) | (two(v.w) << 16));
}
// The same for a power of two: the product of a bf16 value with it is a bf16 value (where it is not, being subnormal, the
// code is zero all the same), so two values take one product.
__device__ __forceinline__ uint2 q8_codes8_pow2(uint4 v, uint32_t inv2) {
    auto two = [&](uint32_t w) {
        uint32_t p;
        asm("mul.rn.bf16x2 %0, %1, %2;\n" : "=r"(p) : "r"(w), "r"(inv2));
        return to_e4m3x2(__uint_as_float(p << 16), __uint_as_float(p & 0xFFFF0000u));
    };
    return make_uint2(two(v.x) | (two(v.y) << 16), two(v.z) | (two(v.w) << 16));
}
__device__ __forceinline__ uint32_t q8_amax8(uint4 v) {
    uint32_t m = 0;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(q8_finite_abs(w[i] << 16), q8_finite_abs(w[i] & 0xFFFF0000u)));
    return m;
}

}  // namespace
