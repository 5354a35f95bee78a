// Rotary positions of packed rows: pair i of a head's rotated part is turned by position * f_i,
//     (u, v) -> (u cos a - v sin a, v cos a + u sin a),     a = position * f_i,
// in fp32 from bf16 inputs, rounded once.  A row's R/2 sines and cosines serve all of its heads, so a CTA computes those of a
// tile of rows into shared memory and walks the tile's 16-byte pieces with them.  Bound by memory: two bytes read and two
// written per element.
#include <algorithm>
#include <cmath>

#include "latent.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTileRows = 8;

// One of the call's two tensors, strides in elements.
struct rope_tensor {
    const __nv_bfloat16* x;
    __nv_bfloat16* out;
    int64_t x_row, x_head, out_row, out_head;
    int heads, head_dim, offset, copies;      // copies: whether the elements that do not turn are copied too
};
struct rope_args {
    const uint64_t* turns;
    const int32_t* positions;
    rope_tensor t[2];
    int rows, R, tile_rows, tensors;
    float amplitude, sign;
};

// Pieces: with VEC eight elements and 16 bytes, else one; a rotated piece of the half layout has its partner R/2 behind it.
template <bool HALF, bool VEC>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ rope_args a) {
    extern __shared__ float2 cs[];            // [tile rows][R / 2]
    constexpr int E = VEC ? 8 : 1;            // elements per piece
    const int half = a.R / 2;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int turning = HALF ? half / E : VEC ? a.R / 8 : half;          // rotated pieces per head
    for (int64_t r0 = (int64_t)blockIdx.x * a.tile_rows; r0 < a.rows; r0 += (int64_t)gridDim.x * a.tile_rows) {
        const int n = (int)min((int64_t)a.tile_rows, a.rows - r0);
        __syncthreads();
        for (int i = threadIdx.x; i < n * half; i += kThreads) {
            const int r = i / half, p = i - r * half;
            float2 v = rope_cos_sin(ld_u64(a.turns + p), ld_i32(a.positions + r0 + r), a.amplitude);
            v.y *= a.sign;
            cs[i] = v;
        }
        __syncthreads();
        for (int which = 0; which < a.tensors; ++which) {
            const rope_tensor& t = a.t[which];
            const int rest = t.copies ? (t.head_dim - a.R) / E : 0, per_head = turning + rest, per_row = t.heads * per_head;
            for (int i = threadIdx.x; i < n * per_row; i += kThreads) {
                const int r = i / per_row, j = i - r * per_row, h = j / per_head, p = j - h * per_head;
                const __nv_bfloat16* x = t.x + (r0 + r) * t.x_row + h * t.x_head;
                __nv_bfloat16* o = t.out + (r0 + r) * t.out_row + h * t.out_head;
                if (p >= turning) {
                    int e = (p - turning) * E;
                    if (e >= t.offset) e += a.R;
                    if (VEC) *reinterpret_cast<uint4*>(o + e) = ld_v4(x + e);
                    else *reinterpret_cast<uint16_t*>(o + e) = (uint16_t)ld_u16(x + e);
                    continue;
                }
                const float2* c = cs + r * half;
                if (HALF) {
                    const int e = t.offset + p * E;
                    if (VEC) {
                        const uint4 u = ld_v4(x + e), v = ld_v4(x + e + half);
                        const uint32_t lo[4] = {u.x, u.y, u.z, u.w}, hi[4] = {v.x, v.y, v.z, v.w};
                        uint32_t ol[4], oh[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float2 c0 = c[p * 8 + 2 * k], c1 = c[p * 8 + 2 * k + 1];
                            const float u0 = bf_lo(lo[k]), u1 = bf_hi(lo[k]), v0 = bf_lo(hi[k]), v1 = bf_hi(hi[k]);
                            ol[k] = bf_pack(turn_first(u0, v0, c0), turn_first(u1, v1, c1));
                            oh[k] = bf_pack(turn_second(u0, v0, c0), turn_second(u1, v1, c1));
                        }
                        *reinterpret_cast<uint4*>(o + e) = make_uint4(ol[0], ol[1], ol[2], ol[3]);
                        *reinterpret_cast<uint4*>(o + e + half) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
                    } else {
                        const uint32_t w = rope_turn(ld_u16(x + e) | ld_u16(x + e + half) << 16, c[p]);
                        *reinterpret_cast<uint16_t*>(o + e) = (uint16_t)w;
                        *reinterpret_cast<uint16_t*>(o + e + half) = (uint16_t)(w >> 16);
                    }
                } else if (VEC) {
                    const int e = t.offset + p * 8;
                    const uint4 u = ld_v4(x + e);
                    *reinterpret_cast<uint4*>(o + e) =
                        make_uint4(rope_turn(u.x, c[p * 4]), rope_turn(u.y, c[p * 4 + 1]), rope_turn(u.z, c[p * 4 + 2]),
                                   rope_turn(u.w, c[p * 4 + 3]));
                } else {
                    const int e = t.offset + p * 2;
                    const uint32_t w = rope_turn(ld_u16(x + e) | ld_u16(x + e + 1) << 16, c[p]);
                    *reinterpret_cast<uint16_t*>(o + e) = (uint16_t)w;
                    *reinterpret_cast<uint16_t*>(o + e + 1) = (uint16_t)(w >> 16);
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
          s->out_row_stride, s->out_head_stride, s->heads, s->head_dim, s->offset, in_place ? 0 : 1};
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
    a.tile_rows = (int)std::min<int64_t>(kMaxTileRows, std::max<int64_t>(1, num_rows / 592));
    const int grid = (int)std::min<int64_t>(((int64_t)num_rows + a.tile_rows - 1) / a.tile_rows, 148 * 8);
    auto kernel = half ? (vec ? rope_kernel<true, true> : rope_kernel<true, false>)
                       : (vec ? rope_kernel<false, true> : rope_kernel<false, false>);
    return q8_launch_smem(kernel, grid, kThreads, a.tile_rows * a.R / 2 * 8, (cudaStream_t)stream, a);
}
