// Decode over the 8-bit cache: one query token per block over that block's pages.
#include "cache_q8.cuh"

namespace {

constexpr int kWarps = 4;

// A block's cached tokens as this launch sees them: what it attends over, or -1 when it sits out.
__device__ __forceinline__ int block_len(int b, const q8_tables& t, const int32_t* __restrict__ lens,
                                         const int32_t* __restrict__ active, bool append, int& status) {
    status = 0;
    if (active && active[b] == 0) return -1;
    const int64_t room = (int64_t)(t.page_indptr[b + 1] - t.page_indptr[b]) * kPage, len = lens[b];
    if (len < 0) status = kStatusInvalid;
    else if (len + append > room) status = kStatusNoSpace;
    return status ? -1 : (int)len + append;
}

// One CTA per (block, kv head); a warp takes every fourth token, a lane D / 32 dimensions.
template <int D>
__global__ void __launch_bounds__(kWarps * 32)
decode_q8_simple_kernel(q8_tables t, const __nv_bfloat16* __restrict__ q, const __nv_bfloat16* __restrict__ k_new,
                        const __nv_bfloat16* __restrict__ v_new, const int32_t* __restrict__ lens,
                        int32_t* __restrict__ lens_out, const int32_t* __restrict__ active, uint8_t* pool, float* scales,
                        __nv_bfloat16* __restrict__ o, int Hq, int Hkv, int G, float scale_log2) {
    constexpr int E = D / 32;
    __shared__ float sm_o[kWarps][8][D], sm_m[kWarps][8], sm_l[kWarps][8];
    const int b = blockIdx.x, g = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int status;
    const int len = block_len(b, t, lens, active, k_new != nullptr, status);
    if (g == 0 && threadIdx.x == 0) {
        if (status) atomicCAS(t.header, 0, status);
        if (lens_out) lens_out[b] = len < 0 ? lens[b] : len;
    }
    if (len < 0) return;
    const int32_t* pages = t.page_indices + t.page_indptr[b];
    if (k_new && warp < 2) {                      // the new row: warp 0 its K, warp 1 its V
        const int pos = len - 1, slot = pos % kPage;
        const int64_t c = (int64_t)pages[pos / kPage] * Hkv + g;
        uint8_t* to = pool + c * (2 * kPage * D) + warp * (kPage * D);
        const __nv_bfloat16* src = (warp ? v_new : k_new) + ((int64_t)b * Hkv + g) * D;
        uint32_t amax = 0;
        for (int i = lane; i < D; i += 32) amax = max(amax, q8_finite_abs(__float_as_uint(__bfloat162float(src[i]))));
        amax = __reduce_max_sync(0xffffffffu, amax);
        float s = q8_scale(amax);
        if (slot > 0) {
            const float old = scales[c * 2 + warp];
            if (s > old) {
                const float f = old * q8_inverse(s);
                for (int i = lane; i < slot * (D / 4); i += 32) {
                    uint32_t* w = reinterpret_cast<uint32_t*>(to) + i;
                    *w = q8_rescale4(*w, f);
                }
            } else {
                s = old;
            }
        }
        __syncwarp();
        if (lane == 0) scales[c * 2 + warp] = s;
        const bool pow2 = (__float_as_uint(s) & 0x807FFFFFu) == 0 && s <= 0x1p120f;
        const float inv = pow2 ? q8_inverse(s) : 1.f / s;
        for (int i = lane; i < D; i += 32) to[slot * D + i] = (uint8_t)to_e4m3x2(mul_keep(__bfloat162float(src[i]), inv), 0.f);
    }
    __syncthreads();
    float qf[8][E], acc[8][E], m[8], l[8];
    for (int h = 0; h < 8; ++h) {
        m[h] = -INFINITY; l[h] = 0.f;
        for (int e = 0; e < E; ++e) {
            qf[h][e] = h < G ? __bfloat162float(q[((int64_t)b * Hq + g * G + h) * D + lane * E + e]) : 0.f;
            acc[h][e] = 0.f;
        }
    }
    for (int j = warp; j < len; j += kWarps) {
        const int64_t c = (int64_t)pages[j / kPage] * Hkv + g;
        const uint8_t* kr = pool + c * (2 * kPage * D) + (j % kPage) * D + lane * E;
        const float ks = scales[c * 2], vs = scales[c * 2 + 1];
        float kf[E], vf[E];
        for (int e = 0; e < E; ++e) {
            kf[e] = e4m3x2_to_f32(kr[e]).x * ks;
            vf[e] = e4m3x2_to_f32(kr[kPage * D + e]).x * vs;
        }
        for (int h = 0; h < G; ++h) {
            float s = 0.f;
            for (int e = 0; e < E; ++e) s = fmaf(qf[h][e], kf[e], s);
            for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
            s *= scale_log2;
            const float mn = fmaxf(m[h], s), f = exp2f(m[h] - mn), p = exp2f(s - mn);
            m[h] = mn;
            l[h] = l[h] * f + p;
            for (int e = 0; e < E; ++e) acc[h][e] = acc[h][e] * f + p * vf[e];
        }
    }
    for (int h = 0; h < G; ++h) {
        if (lane == 0) { sm_m[warp][h] = m[h]; sm_l[warp][h] = l[h]; }
        for (int e = 0; e < E; ++e) sm_o[warp][h][lane * E + e] = acc[h][e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < G * D; i += kWarps * 32) {
        const int h = i / D, d = i % D;
        float mx = -INFINITY, sum = 0.f, out = 0.f;
        for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, sm_m[w][h]);
        for (int w = 0; w < kWarps; ++w) {
            const float f = sm_m[w][h] == -INFINITY ? 0.f : exp2f(sm_m[w][h] - mx);
            sum += f * sm_l[w][h];
            out += f * sm_o[w][h][d];
        }
        o[((int64_t)b * Hq + g * G + h) * D + d] = __float2bfloat16(len == 0 ? 0.f : out / sum);
    }
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int launch(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* q, const void* k_new,
           const void* v_new, const int32_t* d_lens, int32_t* d_lens_out, const int32_t* d_active, void* kv_pool,
           float* kv_scales, void* o, void* d_workspace, void* stream) {
    const int rc = q8_check(cfg, dims);
    if (rc != CPA_OK) return rc;
    if (!d_tables || !q || !d_lens || !kv_pool || !kv_scales || !o || !d_workspace || !cpa_aligned16(d_tables) ||
        !cpa_aligned16(q) || !cpa_aligned16(kv_pool) || !cpa_aligned16(kv_scales) || !cpa_aligned16(o) ||
        !cpa_aligned16(d_workspace) || !aligned4(d_lens) || !aligned4(d_lens_out) || !aligned4(d_active))
        return CPA_EINVAL;
    const q8_tables t = q8_view(*cfg, *dims, d_tables);
    const int G = cfg->num_q_heads / cfg->num_kv_heads;
    auto kernel = cfg->head_dim == 128 ? decode_q8_simple_kernel<128> : decode_q8_simple_kernel<64>;
    kernel<<<dim3(dims->num_blocks, cfg->num_kv_heads), kWarps * 32, 0, (cudaStream_t)stream>>>(
        t, (const __nv_bfloat16*)q, (const __nv_bfloat16*)k_new, (const __nv_bfloat16*)v_new, d_lens, d_lens_out, d_active,
        (uint8_t*)kv_pool, kv_scales, (__nv_bfloat16*)o, cfg->num_q_heads, cfg->num_kv_heads, G,
        cfg->scale * 1.4426950408889634f);
    return cudaGetLastError() == cudaSuccess ? CPA_OK : CPA_ECUDA;
}

}  // namespace

extern "C" int64_t cpa_decode_q8_workspace_bytes(const cpa_config* cfg) {
    const cpa_table_dims one{1, 0, 1, 1, 0};
    const int rc = q8_check(cfg, &one);
    return rc != CPA_OK ? rc : 256;
}

extern "C" int cpa_decode_q8(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* q,
                             const int32_t* d_lens, const int32_t* d_active, const void* kv_pool, const float* kv_scales,
                             void* o, void* d_workspace, void* stream) {
    return launch(cfg, dims, d_tables, q, nullptr, nullptr, d_lens, nullptr, d_active, const_cast<void*>(kv_pool),
                  const_cast<float*>(kv_scales), o, d_workspace, stream);
}

extern "C" int cpa_decode_append_q8(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* q,
                                    const void* k_new, const void* v_new, const int32_t* d_lens, int32_t* d_lens_out,
                                    const int32_t* d_active, void* kv_pool, float* kv_scales, void* o, void* d_workspace,
                                    void* stream) {
    if (!k_new || !v_new || !d_lens_out || d_lens == d_lens_out || !cpa_aligned16(k_new) || !cpa_aligned16(v_new))
        return CPA_EINVAL;
    return launch(cfg, dims, d_tables, q, k_new, v_new, d_lens, d_lens_out, d_active, kv_pool, kv_scales, o, d_workspace,
                  stream);
}
