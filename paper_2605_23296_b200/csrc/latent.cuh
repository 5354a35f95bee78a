// Latent attention and rotary positions: the checks of their configurations and the angle arithmetic that their kernels share.
#pragma once

#include "cache_q8.cuh"

namespace {

constexpr int kRopeDim = 64;                  // rotated part of a latent row
constexpr int kMaxLatent = 512;
constexpr int kMaxLatentHeads = 128;

inline bool rope_config_ok(const cpa_rope_config* r) {
    if (!r || r->rope_dim < 2 || r->rope_dim > 256 || r->rope_dim % 2 != 0) return false;
    if (r->layout != CPA_ROPE_HALF && r->layout != CPA_ROPE_INTERLEAVED) return false;
    if (!(r->base > 0.0) || !(r->base <= 1e30) || !(r->amplitude > 0.0) || !(r->amplitude <= 1e4)) return false;
    if (r->scaling == CPA_ROPE_UNSCALED) return true;
    if (!(r->factor > 0.0) || !(r->factor <= 1e6)) return false;
    if (r->scaling == CPA_ROPE_SCALED_ALL) return true;
    if (r->scaling == CPA_ROPE_SCALED_BASE) return r->rope_dim > 2;
    if (r->scaling != CPA_ROPE_SCALED_PARTS && r->scaling != CPA_ROPE_SCALED_WAVES) return false;
    return r->trained_len >= 1 && r->slow > 0.0 && r->fast > r->slow && r->fast <= 1e9 &&
           (r->scaling != CPA_ROPE_SCALED_PARTS || r->base > 1.0);
}

// CPA_OK, or why the configuration is refused.
inline int latent_check(const cpa_latent_config* c) {
    if (!c || c->num_heads < 1 || c->latent_dim < 1 || c->rope_dim < 1 || c->nope_dim < 1 || c->v_dim < 1 || c->num_sms < 0 ||
        !(c->scale > 0.f) || !(c->scale <= 3e38f) || !(c->norm_eps >= 0.f) || !(c->norm_eps <= 3e38f))
        return CPA_EINVAL;
    if (c->num_heads > kMaxLatentHeads || c->latent_dim % 128 != 0 || c->latent_dim > kMaxLatent || c->rope_dim != kRopeDim ||
        c->nope_dim != 128 || c->v_dim != 128 || c->page_size != kPage || c->num_sms > kMaxPlanSms)
        return CPA_EUNSUPPORTED;
    return CPA_OK;
}
inline cpa_config latent_tables_cfg(const cpa_latent_config& c) {
    cpa_config t = {};
    t.num_q_heads = t.num_kv_heads = 1;
    t.head_dim = 64;
    t.page_size = kPage;
    t.scale = c.scale;
    t.num_sms = c.num_sms;
    return t;
}
inline bool latent_aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The angle of a pair at a position.  `turns` holds the pair's frequency in turns per position as a 64-bit binary fraction,
// so position * turns modulo 2^64 is the angle's fractional part with no error but the fraction's own (2^-64 turns, times the
// position): any int32 position, negative ones too, is reduced exactly by the product's wrap-around.  32 bits of it, as a
// signed fraction of half a turn, go to the sine and cosine.
__device__ __forceinline__ float2 rope_cos_sin(uint64_t turns, int32_t position, float amplitude) {
    const uint64_t a = (uint64_t)(int64_t)position * turns;
    const int32_t t = (int32_t)(uint32_t)((a + 0x80000000ull) >> 32);
    float s, c;
    sincospif((float)t * 0x1p-31f, &s, &c);
    return make_float2(c * amplitude, s * amplitude);
}
__device__ __forceinline__ uint64_t ld_u64(const uint64_t* p) {
    uint64_t v;
    asm volatile("ld.global.u64 %0, [%1];\n" : "=l"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint4 ld_v4(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_u16(const void* p) {
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];\n" : "=h"(v) : "l"(p));
    return v;
}
// eight bf16 values that may lie anywhere
__device__ __forceinline__ uint4 ld_8x16(const __nv_bfloat16* p) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = ld_u16(p + i);
    return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
// a * b + c that keeps subnormals (see mul_keep)
__device__ __forceinline__ float fma_keep(float a, float b, float c) {
    float d;
    asm("fma.rn.f32 %0, %1, %2, %3;\n" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// the two elements of a pair turned by the angle of (cos, sin)
__device__ __forceinline__ float turn_first(float u, float v, float2 cs) { return fma_keep(u, cs.x, -mul_keep(v, cs.y)); }
__device__ __forceinline__ float turn_second(float u, float v, float2 cs) { return fma_keep(v, cs.x, mul_keep(u, cs.y)); }
// the same for a pair in one word, the first element below
__device__ __forceinline__ uint32_t rope_turn(uint32_t w, float2 cs) {
    const float u = bf_lo(w), v = bf_hi(w);
    return bf_pack(turn_first(u, v, cs), turn_second(u, v, cs));
}

}  // namespace

// cpa_latent_append over the blocks whose flag in d_active is not 0 (nullptr: all).
int cpa_latent_append_rows(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables, const cpa_rope_config* rope,
                           const uint64_t* d_turns, const void* x, int64_t x_row_stride, const void* norm_weight,
                           const int32_t* d_cu_new, int32_t num_rows, const int32_t* d_first, const int32_t* d_lens,
                           int32_t* d_lens_out, const int32_t* d_active, void* pool, void* packed, void* stream);
