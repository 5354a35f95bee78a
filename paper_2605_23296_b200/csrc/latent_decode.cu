// Absorbed latent attention of one query token per block over the paged latent cache.
#include <algorithm>

#include "latent.cuh"

namespace {

constexpr int kWarps = 8;

struct decode_args {
    q8_tables t;
    cpa_latent_io io;
    const uint64_t* turns;            // step: the query's positional part is turned; nullptr: taken as it is
    const int32_t *first, *lens, *lens_before, *active;   // lens_before: step, blocks that have not grown sit out
    const __nv_bfloat16* pool;
    int B, H, interleaved;
    float scale, amplitude;
};

// One CTA per (block, head), a warp per token, lanes over the row's 16-byte pieces.
template <int L>
__global__ void __launch_bounds__(kWarps * 32) latent_decode_kernel(const __grid_constant__ decode_args a) {
    constexpr int C = L / 8, N = C + kRopeDim / 8, K = (N + 31) / 32;
    __shared__ float sm_o[kWarps][L], sm_m[kWarps], sm_l[kWarps], sm_rope[kRopeDim];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int b = blockIdx.x / a.H, h = blockIdx.x % a.H;
    const int len = ld_i32(a.lens + b), ip = ld_i32(a.t.page_indptr + b), np = ld_i32(a.t.page_indptr + b + 1) - ip;
    if (a.active && ld_i32(a.active + b) == 0) return;
    if (a.lens_before && ld_i32(a.lens_before + b) == len) return;
    if (len < 0 || len > (int64_t)np * kPage) {
        if (threadIdx.x == 0) atomicCAS(a.t.header, 0, len < 0 ? kStatusInvalid : kStatusNoSpace);
        return;
    }
    const __nv_bfloat16* qc = (const __nv_bfloat16*)a.io.q_latent + b * a.io.q_latent_block_stride + h * a.io.q_latent_head_stride;
    const __nv_bfloat16* qr = (const __nv_bfloat16*)a.io.q_rope + b * a.io.q_rope_block_stride + h * a.io.q_rope_head_stride;
    if (threadIdx.x < 32) {
        const int u = a.interleaved ? 2 * lane : lane, v = a.interleaved ? 2 * lane + 1 : lane + 32;
        uint32_t w = ld_u16(qr + u) | ld_u16(qr + v) << 16;
        if (a.turns) w = rope_turn(w, rope_cos_sin(ld_u64(a.turns + lane), (a.first ? ld_i32(a.first + b) : 0) + len - 1, a.amplitude));
        sm_rope[u] = bf_lo(w);
        sm_rope[v] = bf_hi(w);
    }
    __syncthreads();
    float q[K][8], o[K][8], m = -3e38f, l = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int p = lane + 32 * k;
        const uint4 w = p < C ? ld_v4(qc + 8 * p) : make_uint4(0, 0, 0, 0);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { q[k][2 * i] = bf_lo(ww[i]); q[k][2 * i + 1] = bf_hi(ww[i]); }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (p >= C && p < N) q[k][i] = sm_rope[8 * (p - C) + i];
            o[k][i] = 0.f;
        }
    }
    for (int j = warp; j < len; j += kWarps) {
        const __nv_bfloat16* row = a.pool + ((int64_t)ld_i32(a.t.page_indices + ip + j / kPage) * kPage + j % kPage) * (L + kRopeDim);
        float x[K][8], s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int p = lane + 32 * k;
            const uint4 w = p < N ? ld_v4(row + 8 * p) : make_uint4(0, 0, 0, 0);
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[k][2 * i] = bf_lo(ww[i]); x[k][2 * i + 1] = bf_hi(ww[i]); }
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(q[k][i], x[k][i], s);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= a.scale * 1.4426950408889634f;
        const float m2 = fmaxf(m, s), f = exp2f(m - m2), e = exp2f(s - m2);
        m = m2;
        l = l * f + e;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) o[k][i] = o[k][i] * f + e * x[k][i];
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * k < C) sm_o[warp][8 * (lane + 32 * k) + i] = o[k][i];
    if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
    __syncthreads();
    float mm = -3e38f, ll = 0.f;
    for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sm_m[w]);
    for (int w = 0; w < kWarps; ++w) ll += sm_l[w] * exp2f(sm_m[w] - mm);
    __nv_bfloat16* out = (__nv_bfloat16*)a.io.o + b * a.io.o_block_stride + h * a.io.o_head_stride;
    for (int e = threadIdx.x; e < L; e += kWarps * 32) {
        float v = 0.f;
        for (int w = 0; w < kWarps; ++w) v += sm_o[w][e] * exp2f(sm_m[w] - mm);
        out[e] = __float2bfloat16(len == 0 ? 0.f : v / ll);
    }
}

bool io_ok(const cpa_latent_io* io, int B, int H, int L) {
    if (!io || !io->q_latent || !io->q_rope || !io->o || !latent_aligned(io->q_latent, 16) || !latent_aligned(io->q_rope, 16) ||
        !latent_aligned(io->o, 16))
        return false;
    for (int64_t s : {io->q_latent_block_stride, io->q_latent_head_stride, io->q_rope_block_stride, io->q_rope_head_stride,
                      io->o_block_stride, io->o_head_stride})
        if (s % 8 != 0) return false;
    // heads of the output must not share elements: blocks of heads, or heads of blocks
    const int64_t bs = B > 1 ? io->o_block_stride : INT64_MAX, hs = H > 1 ? io->o_head_stride : INT64_MAX;
    if (bs < L || hs < L) return false;
    return B == 1 || H == 1 || bs >= (H - 1) * hs + L || hs >= (B - 1) * bs + L;
}

int decode(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables, const cpa_rope_config* rope,
           const uint64_t* d_turns, const cpa_latent_io* io, const int32_t* d_first, const int32_t* d_lens,
           const int32_t* d_before, const int32_t* d_active, const void* pool, void* stream) {
    decode_args a = {};
    a.t = q8_view(latent_tables_cfg(*cfg), *dims, d_tables);
    a.io = *io;
    a.turns = d_turns;
    a.first = d_first;
    a.lens = d_lens;
    a.lens_before = d_before;
    a.active = d_active;
    a.pool = (const __nv_bfloat16*)pool;
    a.B = dims->num_blocks;
    a.H = cfg->num_heads;
    a.interleaved = rope && rope->layout == CPA_ROPE_INTERLEAVED;
    a.scale = cfg->scale;
    a.amplitude = rope ? (float)rope->amplitude : 1.f;
    auto kernel = cfg->latent_dim == 128   ? latent_decode_kernel<128>
                  : cfg->latent_dim == 256 ? latent_decode_kernel<256>
                  : cfg->latent_dim == 384 ? latent_decode_kernel<384>
                                           : latent_decode_kernel<512>;
    return q8_launch(kernel, a.B * a.H, kWarps * 32, (cudaStream_t)stream, a);
}

int check(const cpa_latent_config* cfg, const cpa_table_dims* dims, const void* d_tables, const cpa_latent_io* io,
          const int32_t* d_lens, const int32_t* d_active, const void* pool, const void* d_workspace) {
    int rc = latent_check(cfg);
    if (rc != CPA_OK) return rc;
    const cpa_config tc = latent_tables_cfg(*cfg);
    rc = q8_check(&tc, dims);
    if (rc != CPA_OK) return rc;
    if (!d_tables || !d_lens || !pool || !d_workspace || !latent_aligned(d_tables, 16) || !latent_aligned(d_lens, 4) ||
        !latent_aligned(d_active, 4) || !latent_aligned(pool, 16) || !latent_aligned(d_workspace, 16) ||
        !io_ok(io, dims->num_blocks, cfg->num_heads, cfg->latent_dim))
        return CPA_EINVAL;
    return CPA_OK;
}

}  // namespace

extern "C" int64_t cpa_latent_decode_workspace_bytes(const cpa_latent_config* cfg) {
    const int rc = latent_check(cfg);
    return rc != CPA_OK ? rc : 256;
}

extern "C" int cpa_latent_decode(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                                 const cpa_latent_io* io, const int32_t* d_lens, const int32_t* d_active, const void* pool,
                                 void* d_workspace, void* stream) {
    const int rc = check(cfg, dims, d_tables, io, d_lens, d_active, pool, d_workspace);
    if (rc != CPA_OK) return rc;
    return decode(cfg, dims, d_tables, nullptr, nullptr, io, nullptr, d_lens, nullptr, d_active, pool, stream);
}

extern "C" int cpa_latent_step(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                               const cpa_rope_config* rope, const uint64_t* d_turns, const cpa_latent_io* io, const void* x,
                               int64_t x_row_stride, const void* norm_weight, const int32_t* d_first, const int32_t* d_lens,
                               int32_t* d_lens_out, const int32_t* d_active, void* pool, void* d_workspace, void* stream) {
    int rc = check(cfg, dims, d_tables, io, d_lens, d_active, pool, d_workspace);
    if (rc != CPA_OK) return rc;
    if (!d_lens_out) return CPA_EINVAL;
    rc = cpa_latent_append_rows(cfg, dims, d_tables, rope, d_turns, x, x_row_stride, norm_weight, nullptr, dims->num_blocks, d_first,
                                d_lens, d_lens_out, d_active, pool, nullptr, stream);
    if (rc != CPA_OK) return rc;
    return decode(cfg, dims, d_tables, rope, d_turns, io, d_first, d_lens_out, d_lens, d_active, pool, stream);
}
