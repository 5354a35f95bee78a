// Latent rows into the paged cache: of a row x = [latent part | positional part],
//     c = x_c / sqrt(mean(x_c^2) + eps) * weight,      r = x_r turned to the token's position,
// in fp32, rounded once to bf16, to the token's slot and, where asked for, to a packed row.  Bound by memory: 2 (L + 64) bytes
// read and as many (or twice as many) written per token.  One warp takes a row: lane i holds the 16-byte pieces i, i + 32 and
// i + 64 of it, so the sum of squares is a warp's sum, and each lane computes one of the 32 sines and cosines.
#include <algorithm>

#include "latent.cuh"

namespace {

constexpr int kWarps = 8;

struct append_args {
    q8_tables t;
    const __nv_bfloat16* x;
    const __nv_bfloat16* weight;      // nullptr: the latent part is stored as it is
    const uint64_t* turns;            // nullptr: so is the positional part
    const int32_t *cu, *first, *lens; // nullptr: one row per block; 0 everywhere; 0 everywhere
    const int32_t* active;            // nullptr: all blocks; a block with flag 0 is left out, without a status
    int32_t* lens_out;
    __nv_bfloat16 *pool, *packed;
    int64_t x_row;
    int B, rows, interleaved, row_ctas;
    float eps, amplitude;
};

__device__ __forceinline__ int cu_at(const int32_t* cu, int b) { return cu ? ld_i32(cu + b) : b; }

// The last block that starts at or before a packed row, by a whole warp with 32 candidates per load.  What it leads to
// grows with the row, whatever cu holds.
__device__ __forceinline__ int find_block(int row, const int32_t* cu, int B, int lane) {
    if (!cu) return row;
    int lo = 0, size = B;
    while (size > 1) {
        const int step = (size + 31) / 32, i = lane * step;
        const uint32_t below = __ballot_sync(0xffffffffu, i < size && ld_i32(cu + lo + i) <= row);
        const int skip = max(__popc(below) - 1, 0) * step;
        lo += skip;
        size = min(step, size - skip);
    }
    return lo;
}

// A block's rows: n from packed row c0 on, to position `at`; and 0, or the status of why it is left out.
struct block_rows { int c0, n, at, ip, status; };
__device__ __forceinline__ block_rows rows_of(int b, const append_args& a) {
    const int c0 = cu_at(a.cu, b), c1 = cu_at(a.cu, b + 1), at = a.lens ? ld_i32(a.lens + b) : 0;
    const int ip = ld_i32(a.t.page_indptr + b), np = ld_i32(a.t.page_indptr + b + 1) - ip;
    const bool bad = c1 < c0 || at < 0 || c0 < 0 || c1 > a.rows;
    const bool out = a.active && ld_i32(a.active + b) == 0;
    const int n = bad || out ? 0 : c1 - c0;
    if (out) return {c0, 0, at, ip, 0};
    return {c0, n, at, ip, bad ? kStatusInvalid : (int64_t)at + n > (int64_t)np * kPage ? kStatusNoSpace : 0};
}

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
__device__ __forceinline__ void make_row(row_pieces<L>& r, const append_args& a, int position, int lane) {
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

// Packed row `row`, which is row `row - b.c0` of block b, through to its slot.
template <int L>
__device__ __forceinline__ void put_row(row_pieces<L>& r, int row, int block, const block_rows& b, const append_args& a, int lane) {
    const int at = b.at + row - b.c0;
    const int page = ld_i32(a.t.page_indices + b.ip + at / kPage);
    make_row<L>(r, a, (a.first ? ld_i32(a.first + block) : 0) + at, lane);
    store_row<L>(r, a.pool + ((int64_t)page * kPage + at % kPage) * (L + kRopeDim), lane);
    if (a.packed) store_row<L>(r, a.packed + (int64_t)row * (L + kRopeDim), lane);
}

template <int L, bool WIDE>
__global__ void __launch_bounds__(kWarps * 32) latent_append_kernel(const __grid_constant__ append_args a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    row_pieces<L> r;
    if ((int)blockIdx.x >= a.row_ctas) {          // the blocks' books, a warp each
        for (int64_t b = (int64_t)((int)blockIdx.x - a.row_ctas) * kWarps + warp; b < a.B; b += (int64_t)(gridDim.x - a.row_ctas) * kWarps) {
            const block_rows o = rows_of((int)b, a);
            if (lane == 0) {
                if (o.status) atomicCAS(a.t.header, 0, o.status);
                if (a.lens_out) a.lens_out[b] = o.at + (o.status ? 0 : o.n);
            }
            if (o.status || o.n == 0 || !a.cu) continue;
            // Where a range runs backwards the search may lead from a good block's rows elsewhere: those are taken here.
            // (What the search leads to grows with the row, so a block's first and last one tell.)
            if (find_block(o.c0, a.cu, a.B, lane) == b && find_block(o.c0 + o.n - 1, a.cu, a.B, lane) == b) continue;
            for (int row = o.c0; row < o.c0 + o.n; ++row) {
                load_row<L, WIDE>(r, a.x + row * a.x_row, lane);
                put_row<L>(r, row, (int)b, o, a, lane);
            }
        }
        return;
    }
    for (int64_t row = (int64_t)blockIdx.x * kWarps + warp; row < a.rows; row += (int64_t)a.row_ctas * kWarps) {
        load_row<L, WIDE>(r, a.x + row * a.x_row, lane);
        const int b = find_block((int)row, a.cu, a.B, lane);
        const block_rows o = rows_of(b, a);
        if (!o.status && row >= o.c0 && row < o.c0 + o.n) put_row<L>(r, (int)row, b, o, a, lane);
    }
}

template <int L>
int launch(const append_args& a, bool wide, int grid, cudaStream_t st) {
    return q8_launch(wide ? latent_append_kernel<L, true> : latent_append_kernel<L, false>, grid, kWarps * 32, st, a);
}

}  // namespace

extern "C" int cpa_latent_tables_config(const cpa_latent_config* cfg, cpa_config* out) {
    const int rc = latent_check(cfg);
    if (rc != CPA_OK || !out) return rc != CPA_OK ? rc : CPA_EINVAL;
    *out = latent_tables_cfg(*cfg);
    return CPA_OK;
}

int cpa_latent_append_rows(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                                 const cpa_rope_config* rope, const uint64_t* d_turns, const void* x, int64_t x_row_stride,
                                 const void* norm_weight, const int32_t* d_cu_new, int32_t num_rows, const int32_t* d_first,
                                 const int32_t* d_lens, int32_t* d_lens_out, const int32_t* d_active, void* pool, void* packed, void* stream) {
    int rc = latent_check(cfg);
    if (rc != CPA_OK) return rc;
    const cpa_config tc = latent_tables_cfg(*cfg);
    rc = q8_check(&tc, dims);
    if (rc != CPA_OK) return rc;
    const int row = cfg->latent_dim + kRopeDim;
    if (!d_tables || num_rows < 0 || (num_rows > 0 && !x) || !pool || !latent_aligned(d_tables, 16) || !latent_aligned(x, 2) ||
        !latent_aligned(norm_weight, 16) || !latent_aligned(pool, 16) || !latent_aligned(packed, 16) || !latent_aligned(d_turns, 8) ||
        !latent_aligned(d_cu_new, 4) || !latent_aligned(d_first, 4) || !latent_aligned(d_lens, 4) || !latent_aligned(d_lens_out, 4) ||
        !latent_aligned(d_active, 4) || (d_lens && d_lens == d_lens_out) || (d_turns != nullptr) != (rope != nullptr))
        return CPA_EINVAL;
    if (rope && (!rope_config_ok(rope) || rope->rope_dim != kRopeDim)) return CPA_EINVAL;
    if (!d_cu_new && num_rows != dims->num_blocks) return CPA_EINVAL;
    if (num_rows > 1 && x_row_stride < row) return CPA_EINVAL;
    append_args a = {};
    a.t = q8_view(tc, *dims, d_tables);
    a.x = (const __nv_bfloat16*)x;
    a.weight = (const __nv_bfloat16*)norm_weight;
    a.turns = d_turns;
    a.cu = d_cu_new;
    a.first = d_first;
    a.lens = d_lens;
    a.active = d_active;
    a.lens_out = d_lens_out;
    a.pool = (__nv_bfloat16*)pool;
    a.packed = (__nv_bfloat16*)packed;
    a.x_row = x_row_stride;
    a.B = dims->num_blocks;
    a.rows = num_rows;
    a.interleaved = rope && rope->layout == CPA_ROPE_INTERLEAVED;
    a.eps = cfg->norm_eps;
    a.amplitude = rope ? (float)rope->amplitude : 1.f;
    a.row_ctas = (int)std::min<int64_t>(((int64_t)num_rows + kWarps - 1) / kWarps, 1 << 20);
    const int grid = a.row_ctas + std::min((a.B + kWarps - 1) / kWarps, 1 << 16);
    const bool wide = latent_aligned(x, 16) && x_row_stride % 8 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    switch (cfg->latent_dim) {
        case 128: return launch<128>(a, wide, grid, st);
        case 256: return launch<256>(a, wide, grid, st);
        case 384: return launch<384>(a, wide, grid, st);
        default: return launch<512>(a, wide, grid, st);
    }
}

extern "C" int cpa_latent_append(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                                 const cpa_rope_config* rope, const uint64_t* d_turns, const void* x, int64_t x_row_stride,
                                 const void* norm_weight, const int32_t* d_cu_new, int32_t num_rows, const int32_t* d_first,
                                 const int32_t* d_lens, int32_t* d_lens_out, void* pool, void* packed, void* stream) {
    return cpa_latent_append_rows(cfg, dims, d_tables, rope, d_turns, x, x_row_stride, norm_weight, d_cu_new, num_rows, d_first,
                                  d_lens, d_lens_out, nullptr, pool, packed, stream);
}
