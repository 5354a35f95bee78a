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
    if (!(r->base > 0.0) || !(r->base <= 1e30) || !(r->amplitude >= 1e-30) || !(r->amplitude <= 1e4)) return false;
    if (r->scaling == CPA_ROPE_UNSCALED) return true;
    if (!(r->factor > 0.0) || !(r->factor <= 1e6)) return false;
    if (r->scaling == CPA_ROPE_SCALED_ALL) return true;
    if (r->scaling == CPA_ROPE_SCALED_BASE) return r->rope_dim > 2;
    if (r->scaling != CPA_ROPE_SCALED_PARTS && r->scaling != CPA_ROPE_SCALED_WAVES) return false;
    return r->trained_len >= 1 && r->slow > 0.0 && r->fast > r->slow && r->fast <= 1e9 &&
           (r->scaling != CPA_ROPE_SCALED_PARTS || r->base > 1.0);
}

// CPA_OK, or why the configuration is refused.  (The scale's range: the kernels multiply with scale * log2(e), which has to be a normal
// number, and flush scores below 2^-126 ahead of it, which are nothing after it up to 2^100.)
inline int latent_check(const cpa_latent_config* c) {
    if (!c || c->num_heads < 1 || c->latent_dim < 1 || c->rope_dim < 1 || c->nope_dim < 1 || c->v_dim < 1 || c->num_sms < 0 ||
        !(c->scale >= 0x1p-100f) || !(c->scale <= 0x1p100f) || !(c->norm_eps >= 0.f) || !(c->norm_eps <= 3e38f))
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
// signed fraction of half a turn, are rounded to fp32 (off by 2^-26 turns at most) and go to the sine and cosine.
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

// ---------------------------------------------------------------- one latent row, by a warp
// How a row becomes a cached one.
struct row_recipe {
    const __nv_bfloat16* weight;      // nullptr: the latent part is stored as it is
    const uint64_t* turns;            // nullptr: so is the positional part
    float eps, amplitude;
    int interleaved;
};
// One row's pieces of a lane.
template <int L> struct row_pieces {
    static constexpr int C = L / 8, N = C + kRopeDim / 8, K = (N + 31) / 32;   // pieces of the latent part, of the row; per lane
    uint4 v[K];
};
template <int L, bool WIDE>
__device__ __forceinline__ void load_row(row_pieces<L>& r, const __nv_bfloat16* x, int lane) {
#pragma unroll
    for (int k = 0; k < row_pieces<L>::K; ++k) {
        const int p = lane + 32 * k;
        r.v[k] = make_uint4(0, 0, 0, 0);
        if (p < row_pieces<L>::N) r.v[k] = WIDE ? ld_v4(x + 8 * p) : ld_8x16(x + 8 * p);
    }
}
// The row as it is cached, in place.
template <int L>
__device__ __forceinline__ void make_row(row_pieces<L>& r, const row_recipe& a, int position, int lane) {
    constexpr int C = row_pieces<L>::C, K = row_pieces<L>::K;
    if (a.weight) {
        float ss = 0.f;
        auto add = [&](const uint4& v, float f) {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = bf_lo(w[i]) * f, hi = bf_hi(w[i]) * f;
                ss = fmaf(lo, lo, fmaf(hi, hi, ss));
            }
        };
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (lane + 32 * k < C) add(r.v[k], 1.f);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        float pre = 1.f, inv = rsqrtf(ss * (1.f / L) + a.eps);
        // squares beyond fp32's range, or below it where nothing is added to them: taken of the row over a power of two
        if (!(ss <= 1e37f) || (ss < 1e-30f && a.eps < 1e-30f)) {
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (lane + 32 * k < C) top = max(top, q8_amax8(r.v[k]));
            top = __reduce_max_sync(0xffffffffu, top);
            const int e = min(max((int)(max(top, __float_as_uint(sqrtf(a.eps))) >> 23), 1), 253);
            pre = __uint_as_float((uint32_t)(254 - e) << 23);      // 2^(127 - e)
            ss = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (lane + 32 * k < C) {
                    const uint32_t w[4] = {r.v[k].x, r.v[k].y, r.v[k].z, r.v[k].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float lo = mul_keep(bf_lo(w[i]), pre), hi = mul_keep(bf_hi(w[i]), pre);
                        ss = fmaf(lo, lo, fmaf(hi, hi, ss));
                    }
                }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            inv = rsqrtf(ss * (1.f / L) + mul_keep(mul_keep(a.eps, pre), pre));
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int p = lane + 32 * k;
            if (p >= C) continue;
            const uint4 g = ld_v4(a.weight + 8 * p);
            auto two = [&](uint32_t x, uint32_t w) {
                return bf_pack(mul_keep(mul_keep(mul_keep(bf_lo(x), pre), inv), bf_lo(w)),
                               mul_keep(mul_keep(mul_keep(bf_hi(x), pre), inv), bf_hi(w)));
            };
            r.v[k] = make_uint4(two(r.v[k].x, g.x), two(r.v[k].y, g.y), two(r.v[k].z, g.z), two(r.v[k].w, g.w));
        }
    }
    if (a.turns) {
        constexpr int k = C / 32;                        // the pieces behind the latent part are all in this round
        static_assert(C % 32 + kRopeDim / 8 <= 32, "");
        const float2 cs = rope_cos_sin(ld_u64(a.turns + lane), position, a.amplitude);     // pair `lane`
        const int p = lane + 32 * k - C;                 // piece of the positional part, where 0 <= p < 8
        uint32_t w[4] = {r.v[k].x, r.v[k].y, r.v[k].z, r.v[k].w};
        auto pair = [&](int i) {
            return make_float2(__shfl_sync(0xffffffffu, cs.x, i & 31), __shfl_sync(0xffffffffu, cs.y, i & 31));
        };
        if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 c = pair(4 * p + i);
                w[i] = rope_turn(w[i], c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {                // the partner's elements are in the lane four on (or back)
                const uint32_t other = __shfl_xor_sync(0xffffffffu, w[i], 4);
                const float2 c0 = pair(8 * p + 2 * i), c1 = pair(8 * p + 2 * i + 1);
                w[i] = (p & 4) ? bf_pack(turn_second(bf_lo(other), bf_lo(w[i]), c0), turn_second(bf_hi(other), bf_hi(w[i]), c1))
                               : bf_pack(turn_first(bf_lo(w[i]), bf_lo(other), c0), turn_first(bf_hi(w[i]), bf_hi(other), c1));
            }
        }
        if (p >= 0 && p < kRopeDim / 8) r.v[k] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <int L>
__device__ __forceinline__ void store_row(const row_pieces<L>& r, __nv_bfloat16* to, int lane) {
#pragma unroll
    for (int k = 0; k < row_pieces<L>::K; ++k) {
        const int p = lane + 32 * k;
        if (p < row_pieces<L>::N) *reinterpret_cast<uint4*>(to + 8 * p) = r.v[k];
    }
}
// The row x, wherever it lies, to `to`.
template <int L>
__device__ __forceinline__ void put_new_row(const __nv_bfloat16* x, const row_recipe& a, int position, __nv_bfloat16* to, int lane) {
    row_pieces<L> r;
    if (__cvta_generic_to_global(x) % 16 == 0) load_row<L, true>(r, x, lane);
    else load_row<L, false>(r, x, lane);
    make_row<L>(r, a, position, lane);
    store_row<L>(r, to, lane);
}

// One lane of the warp, chosen in the form that lets the compiler keep the operands of what that lane runs on the uniform
// datapath: an MMA of 64 x 64 x 16 then goes out every 32 cycles, which is what its operands take out of shared memory, and
// every 46 under a test of the lane's number (58 with the instruction alone predicated on it).  For the same mask it is always the same
// lane, so that a commit from it follows all of its warp's products.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(p));
    return p != 0;
}

}  // namespace
