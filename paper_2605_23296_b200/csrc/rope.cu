// Rotary positions of packed rows: pair i of a head's rotated part is turned by position * f_i,
//     (u, v) -> (u cos a - v sin a, v cos a + u sin a),     a = position * f_i,
// in fp32 from bf16 inputs, rounded once.  A row's R/2 sines and cosines serve all of its heads, so a CTA computes those of a
// tile of rows into shared memory and walks the tile's 16-byte pieces with them.  Bound by memory: two bytes read and two
// written per element.  Measured: 32 + 8 heads of 128 over 32 prompts of 1024..8192 tokens, 2.5 GB, 398 us in a row = 96 % of the
// copy rate (403 to 433 by single calls); one token for each of 192 blocks 2.8 us on the device.  By element, which only shapes that
// hold no 16-byte pieces need, 32 + 8 heads of 80 with 20 rotated elements over the same prompts: 1.23 ms, 1.3 TB/s (16 of 80 by
// pieces 321 us).
#include <algorithm>
#include <cmath>

#include "latent.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kTileRows = 16, kLoneTileRows = 32;
constexpr int kCtas = 4 * 148;                // resident at a time on a B200
constexpr int kBatch = 4;                     // pieces of a thread in flight

// n / d for n < 2^31 by a product: m = ceil(2^(31 + s) / d) with 2^s >= d, whose excess over the true factor is below
// d / 2^(31 + s) <= 2^-31, so n times it never reaches the next whole number.
struct divisor { uint32_t m, s, d; };
divisor make_divisor(uint32_t d) {
    uint32_t s = 0;
    while ((1u << s) < d) ++s;
    return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s, d};
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const divisor& v) { return (uint32_t)((uint64_t)n * v.m >> 31 >> v.s); }

// One of the call's two tensors, strides in elements.
struct rope_tensor {
    const __nv_bfloat16* x;
    __nv_bfloat16* out;
    int64_t x_row, x_head, out_row, out_head;
    int heads, head_dim, offset, copies;      // copies: whether the elements that do not turn are copied too
    divisor per_row, per_head;                // pieces
};
struct rope_args {
    const uint64_t* turns;
    const int32_t* positions;
    rope_tensor t[2];
    int rows, R, tile_rows, tensors, turning; // turning: rotated pieces per head
    divisor half;
    float amplitude, sign;
};

__device__ __forceinline__ uint4 ld_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// Pieces: with VEC eight elements and 16 bytes, else one; a rotated piece of the half layout has its partner R/2 behind it.
template <bool VEC> struct piece { using type = uint4; };
template <> struct piece<false> { using type = uint32_t; };
template <bool VEC> __device__ __forceinline__ typename piece<VEC>::type load_piece(const __nv_bfloat16* p);
template <> __device__ __forceinline__ uint4 load_piece<true>(const __nv_bfloat16* p) { return ld_once(p); }
template <> __device__ __forceinline__ uint32_t load_piece<false>(const __nv_bfloat16* p) { return ld_u16(p); }
__device__ __forceinline__ void store_piece(__nv_bfloat16* p, const uint4& v) { *reinterpret_cast<uint4*>(p) = v; }
__device__ __forceinline__ void store_piece(__nv_bfloat16* p, uint32_t v) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)v; }

__device__ __forceinline__ void turn_halves(uint4& lo, uint4& hi, const float2* c) {
    uint32_t u[4] = {lo.x, lo.y, lo.z, lo.w}, v[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float4 cc = *reinterpret_cast<const float4*>(c + 2 * k);
        const float2 c0 = make_float2(cc.x, cc.y), c1 = make_float2(cc.z, cc.w);
        const float u0 = bf_lo(u[k]), u1 = bf_hi(u[k]), v0 = bf_lo(v[k]), v1 = bf_hi(v[k]);
        u[k] = bf_pack(turn_first(u0, v0, c0), turn_first(u1, v1, c1));
        v[k] = bf_pack(turn_second(u0, v0, c0), turn_second(u1, v1, c1));
    }
    lo = make_uint4(u[0], u[1], u[2], u[3]);
    hi = make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void turn_halves(uint32_t& lo, uint32_t& hi, const float2* c) {
    const uint32_t w = rope_turn(lo | hi << 16, *c);
    lo = w & 0xFFFFu;
    hi = w >> 16;
}
__device__ __forceinline__ void turn_pairs(uint4& v, const float2* c) {
    const float4 a = *reinterpret_cast<const float4*>(c), b = *reinterpret_cast<const float4*>(c + 2);
    v = make_uint4(rope_turn(v.x, make_float2(a.x, a.y)), rope_turn(v.y, make_float2(a.z, a.w)), rope_turn(v.z, make_float2(b.x, b.y)),
                   rope_turn(v.w, make_float2(b.z, b.w)));
}

template <bool HALF, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) rope_kernel(const __grid_constant__ rope_args a) {
    extern __shared__ __align__(16) float2 cs[];          // [tile rows][R / 2]
    constexpr int E = VEC ? 8 : 1;                        // elements per piece
    constexpr bool TWO = HALF || !VEC;                    // a rotated item has two pieces: its partner's too
    const int half = a.R / 2, partner = HALF ? half : 1;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    for (int64_t r0 = (int64_t)blockIdx.x * a.tile_rows; r0 < a.rows; r0 += (int64_t)gridDim.x * a.tile_rows) {
        const int n = (int)min((int64_t)a.tile_rows, a.rows - r0);
        __syncthreads();
        for (int i = threadIdx.x; i < n * half; i += kThreads) {
            const int r = (int)divide(i, a.half), p = i - r * half;
            float2 v = rope_cos_sin(ld_u64(a.turns + p), ld_i32(a.positions + r0 + r), a.amplitude);
            v.y *= a.sign;
            cs[i] = v;
        }
        __syncthreads();
        for (int which = 0; which < a.tensors; ++which) {
            const rope_tensor& t = a.t[which];
            const int per_row = (int)t.per_row.d, per_head = (int)t.per_head.d, total = n * per_row;
            // item i of the tile: elements `e` (and e + partner) of a head, turned by cs[c ...], or copied where c < 0
            struct item { const __nv_bfloat16* x; __nv_bfloat16* o; int c; };
            auto find = [&](int i) {
                const int r = (int)divide(i, t.per_row), j = i - r * per_row, h = (int)divide(j, t.per_head), p = j - h * per_head;
                int e, c = -1;
                if (p < a.turning) {
                    e = t.offset + (HALF ? p * E : VEC ? p * 8 : p * 2);
                    c = r * half + (HALF ? p * E : VEC ? p * 4 : p);
                } else {
                    e = (p - a.turning) * E;
                    if (e >= t.offset) e += a.R;
                }
                return item{t.x + (r0 + r) * t.x_row + h * t.x_head + e, t.out + (r0 + r) * t.out_row + h * t.out_head + e, c};
            };
            for (int i0 = threadIdx.x; i0 < total; i0 += kThreads * kBatch) {
                item it[kBatch];
                typename piece<VEC>::type u[kBatch], v[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const int i = i0 + k * kThreads;
                    if (i >= total) continue;
                    it[k] = find(i);
                    u[k] = load_piece<VEC>(it[k].x);
                    if (TWO && it[k].c >= 0) v[k] = load_piece<VEC>(it[k].x + partner);
                }
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    if (i0 + k * kThreads >= total) continue;
                    if (it[k].c >= 0) {
                        if constexpr (TWO) {
                            turn_halves(u[k], v[k], cs + it[k].c);
                            store_piece(it[k].o + partner, v[k]);
                        } else {
                            turn_pairs(u[k], cs + it[k].c);
                        }
                    }
                    store_piece(it[k].o, u[k]);
                }
            }
        }
    }
}

// Whether the tensor can be walked in 16-byte pieces.
bool pieces_of_16(const rope_tensor& t, int R, bool half_layout) {
    return R % (half_layout ? 16 : 8) == 0 && t.offset % 8 == 0 && t.head_dim % 8 == 0 && t.x_row % 8 == 0 && t.x_head % 8 == 0 &&
           t.out_row % 8 == 0 && t.out_head % 8 == 0 && latent_aligned(t.x, 16) && latent_aligned(t.out, 16);
}

// CPA_OK, or why the tensor is refused.
int make_tensor(const cpa_rope_rows* s, int R, int64_t rows, rope_tensor* t) {
    if (s->heads < 0 || s->head_dim < R || s->offset < 0 || s->offset > s->head_dim - R) return CPA_EINVAL;
    if (s->heads > 65536 || s->head_dim > 65536) return CPA_EUNSUPPORTED;
    if (s->heads == 0 || rows == 0) {
        t->heads = 0;
        return CPA_OK;
    }
    if (!s->x || !s->out || !latent_aligned(s->x, 2) || !latent_aligned(s->out, 2)) return CPA_EINVAL;
    const bool in_place = s->x == s->out;
    if (in_place && (s->x_row_stride != s->out_row_stride || s->x_head_stride != s->out_head_stride)) return CPA_EINVAL;
    // the output's heads and rows may not share elements (one head's stride does not matter, nor one row's)
    const int64_t hs = s->heads > 1 ? s->out_head_stride : s->head_dim, rs = rows > 1 ? s->out_row_stride : 0;
    if (hs < s->head_dim || (rows > 1 && rs < s->head_dim)) return CPA_EINVAL;
    if (rows > 1 && rs < (s->heads - 1) * hs + s->head_dim && hs < (rows - 1) * rs + s->head_dim) return CPA_EINVAL;
    *t = {static_cast<const __nv_bfloat16*>(s->x), static_cast<__nv_bfloat16*>(s->out), s->x_row_stride, s->x_head_stride,
          s->out_row_stride, s->out_head_stride, s->heads, s->head_dim, s->offset, in_place ? 0 : 1, {}, {}};
    return CPA_OK;
}

}  // namespace

extern "C" int cpa_rope_turns(const cpa_rope_config* cfg, uint64_t* turns) {
    if (!rope_config_ok(cfg) || !turns) return CPA_EINVAL;
    const int n = cfg->rope_dim / 2;
    const long double R = cfg->rope_dim, two_pi = 6.283185307179586476925286766559006L;
    long double base = cfg->base;
    if (cfg->scaling == CPA_ROPE_SCALED_BASE) base *= powl((long double)cfg->factor, R / (R - 2));
    // the pair at which `turns` rotations fit into the trained length (SCALED_PARTS)
    auto pair_at = [&](double t) { return R * logl(cfg->trained_len / (two_pi * t)) / (2 * logl(base)); };
    long double lo = 0, hi = 0;
    if (cfg->scaling == CPA_ROPE_SCALED_PARTS) {
        lo = std::max(floorl(pair_at(cfg->fast)), 0.0L);
        hi = std::min(ceill(pair_at(cfg->slow)), R - 1);
    }
    for (int i = 0; i < n; ++i) {
        long double f = powl(base, -2 * i / R);
        long double keep = 1;               // share of the frequency that is not divided by the factor
        if (cfg->scaling == CPA_ROPE_SCALED_ALL) keep = 0;
        if (cfg->scaling == CPA_ROPE_SCALED_PARTS)
            keep = 1 - std::min(std::max((i - lo) / std::max(hi - lo, 0.001L), 0.0L), 1.0L);
        if (cfg->scaling == CPA_ROPE_SCALED_WAVES)
            keep = std::min(std::max((cfg->trained_len * f / two_pi - cfg->slow) / ((long double)cfg->fast - cfg->slow), 0.0L), 1.0L);
        if (keep < 1) f = f * keep + f / (long double)cfg->factor * (1 - keep);
        f /= two_pi;
        f -= floorl(f);                      // whole turns a position do not matter
        const long double scaled = roundl(f * 18446744073709551616.0L);
        turns[i] = scaled >= 18446744073709551616.0L ? 0 : (uint64_t)scaled;
    }
    return CPA_OK;
}

extern "C" int cpa_rope(const cpa_rope_config* cfg, const uint64_t* d_turns, const int32_t* d_positions, int32_t num_rows,
                        const cpa_rope_rows* q, const cpa_rope_rows* k, int inverse, void* stream) {
    if (!rope_config_ok(cfg) || !d_turns || num_rows < 0 || !q || (num_rows > 0 && !d_positions) || !latent_aligned(d_turns, 8) ||
        !latent_aligned(d_positions, 4))
        return CPA_EINVAL;
    rope_args a = {};
    int64_t elements = 0;
    const bool half = cfg->layout == CPA_ROPE_HALF;
    bool vec = true;
    for (const cpa_rope_rows* s : {q, k}) {
        if (!s) continue;
        rope_tensor t = {};
        const int rc = make_tensor(s, cfg->rope_dim, num_rows, &t);
        if (rc != CPA_OK) return rc;
        if (t.heads == 0) continue;
        vec = vec && pieces_of_16(t, cfg->rope_dim, half);
        elements += (int64_t)t.heads * t.head_dim;
        a.t[a.tensors++] = t;
    }
    if (num_rows == 0 || a.tensors == 0) return CPA_OK;
    if (elements > (1 << 24)) return CPA_EUNSUPPORTED;    // a tile's pieces are counted in 32 bits
    a.turns = d_turns;
    a.positions = d_positions;
    a.rows = num_rows;
    a.R = cfg->rope_dim;
    a.amplitude = (float)cfg->amplitude;
    a.sign = inverse ? -1.f : 1.f;
    // Rows per tile: one round of tiles while they have at most kLoneTileRows, else full rounds of at most kTileRows.  (32 + 8 heads of
    // 128: 12000 rows 44 us in a round of 21 rows each, 46 in two; 122,000 rows 398 us in rounds of 16, 414 of 32.  Tiles of 16 in
    // rounds that are not full, 45 of 592 CTAs with a second tile: 8280 rows 38 us for 31.)
    const int64_t rounds = num_rows <= kCtas * kLoneTileRows ? 1 : ((int64_t)num_rows + kCtas * kTileRows - 1) / (kCtas * kTileRows);
    a.tile_rows = (int)((num_rows + kCtas * rounds - 1) / (kCtas * rounds));
    const int E = vec ? 8 : 1;
    a.turning = half ? a.R / 2 / E : vec ? a.R / 8 : a.R / 2;
    a.half = make_divisor((uint32_t)a.R / 2);
    for (int i = 0; i < a.tensors; ++i) {
        rope_tensor& t = a.t[i];
        const uint32_t per_head = (uint32_t)(a.turning + (t.copies ? (t.head_dim - a.R) / E : 0));
        t.per_head = make_divisor(per_head);
        t.per_row = make_divisor(per_head * (uint32_t)t.heads);
    }
    const int grid = (int)std::min<int64_t>(((int64_t)num_rows + a.tile_rows - 1) / a.tile_rows, kCtas);
    auto kernel = half ? (vec ? rope_kernel<true, true> : rope_kernel<true, false>)
                       : (vec ? rope_kernel<false, true> : rope_kernel<false, false>);
    return q8_launch_smem(kernel, grid, kThreads, a.tile_rows * a.R / 2 * 8, (cudaStream_t)stream, a);
}
