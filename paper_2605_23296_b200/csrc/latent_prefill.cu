// Expanded latent attention: causal prefill with keys [k_nope | r], r shared by the heads, on a plan's blocks.
#include "latent.cuh"

namespace {

// One warp per (query row, head), lanes over the head's elements.
__global__ void __launch_bounds__(128) latent_prefill_kernel(const __nv_bfloat16* q, const __nv_bfloat16* kv, const __nv_bfloat16* kr,
                                                             int64_t kr_row, __nv_bfloat16* out, cpa_dev_index ix, int B, int H,
                                                             int tokens, float scale_log2) {
    const int lane = threadIdx.x & 31, i = blockIdx.x * 4 + (threadIdx.x >> 5), h = blockIdx.y;
    if (i >= tokens) return;
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (ld_i32(ix.cu_seqlens + mid) <= i) lo = mid; else hi = mid - 1;
    }
    const int j0 = ld_i32(ix.cu_seqlens + lo);
    const __nv_bfloat16* qi = q + ((int64_t)i * H + h) * 192;
    float a[6], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -3e38f, l = 0.f;
    for (int e = 0; e < 4; ++e) a[e] = __bfloat162float(qi[lane * 4 + e]);
    for (int e = 0; e < 2; ++e) a[4 + e] = __bfloat162float(qi[128 + lane * 2 + e]);
    for (int j = j0; j <= i; ++j) {
        const __nv_bfloat16* kj = kv + ((int64_t)j * H + h) * 256;
        const uint2 k = *reinterpret_cast<const uint2*>(kj + lane * 4), v = *reinterpret_cast<const uint2*>(kj + 128 + lane * 4);
        const uint32_t r = *reinterpret_cast<const uint32_t*>(kr + j * kr_row + lane * 2);
        float s = a[0] * bf_lo(k.x) + a[1] * bf_hi(k.x) + a[2] * bf_lo(k.y) + a[3] * bf_hi(k.y) + a[4] * bf_lo(r) + a[5] * bf_hi(r);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= scale_log2;
        const float m2 = fmaxf(m, s), f = exp2f(m - m2), e = exp2f(s - m2);
        m = m2;
        l = l * f + e;
        o[0] = o[0] * f + e * bf_lo(v.x);
        o[1] = o[1] * f + e * bf_hi(v.x);
        o[2] = o[2] * f + e * bf_lo(v.y);
        o[3] = o[3] * f + e * bf_hi(v.y);
    }
    const float inv = 1.f / l;
    *reinterpret_cast<uint2*>(out + ((int64_t)i * H + h) * 128 + lane * 4) =
        make_uint2(bf_pack(o[0] * inv, o[1] * inv), bf_pack(o[2] * inv, o[3] * inv));
}

}  // namespace

extern "C" int cpa_latent_plan_config(const cpa_latent_config* cfg, cpa_config* out) {
    const int rc = latent_check(cfg);
    if (rc != CPA_OK || !out) return rc != CPA_OK ? rc : CPA_EINVAL;
    *out = {};
    out->num_q_heads = out->num_kv_heads = cfg->num_heads;
    out->head_dim = cfg->v_dim;
    out->page_size = cfg->page_size;
    out->scale = cfg->scale;
    out->num_sms = cfg->num_sms;
    return CPA_OK;
}

extern "C" int cpa_latent_prefill(const cpa_latent_config* cfg, const cpa_plan* plan, const void* q, const void* kv,
                                  const void* k_rope, int64_t k_rope_row_stride, void* o, void* stream) {
    const int rc = latent_check(cfg);
    if (rc != CPA_OK) return rc;
    if (!plan || !q || !kv || !k_rope || !o || !cpa_aligned16(q) || !cpa_aligned16(kv) || !cpa_aligned16(k_rope) ||
        !cpa_aligned16(o) || k_rope_row_stride < kRopeDim || k_rope_row_stride % 8 != 0 || o == q || o == kv || o == k_rope)
        return CPA_EINVAL;
    const cpa_config& c = plan->cfg;
    if (c.num_q_heads != cfg->num_heads || c.num_kv_heads != cfg->num_heads || c.head_dim != cfg->v_dim || c.scale != cfg->scale)
        return CPA_EINVAL;
    for (int32_t p : plan->prefix_lens)
        if (p != 0) return CPA_EUNSUPPORTED;
    if (plan->q_tile == 512) return CPA_EUNSUPPORTED;
    if (!plan->d_base) return CPA_ESTATE;
    const dim3 grid((unsigned)((plan->total_tokens + 3) / 4), (unsigned)cfg->num_heads);
    latent_prefill_kernel<<<grid, 128, 0, (cudaStream_t)stream>>>(
        (const __nv_bfloat16*)q, (const __nv_bfloat16*)kv, (const __nv_bfloat16*)k_rope, k_rope_row_stride, (__nv_bfloat16*)o,
        plan->dev(), plan->B, cfg->num_heads, (int)plan->total_tokens, cfg->scale * 1.4426950408889634f);
    return cudaGetLastError() == cudaSuccess ? CPA_OK : CPA_ECUDA;
}
