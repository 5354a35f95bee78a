// Decode over the 8-bit cache: one query token per block over that block's pages, with the step's append fused in.
//
//   O[h] = sum_j p_j v_j / sum_j p_j,   p_j = 2^(s_j - m),   s_j = scale log2(e) q[h].k_j,   k, v = code * page scale
//
// The step reads every code once (2 bytes per token, kv head and dimension) and is bound by HBM.  Per SM that is a page
// of one kv head (16 tokens, 4 KB at head_dim 128) every 90 ns, so the arithmetic per page has to stay below that:
//   - codes go to the warp-level MMA (m16n8k16, f16 in, fp32 sums) as f16, which holds an e4m3 value exactly; the page
//     scale of K multiplies the finished score.  The queries are made f16 by a power of two per head, exactly but for
//     elements 2^-22 of the row's largest.  (The tensor cores of the fifth generation would take the codes as they are,
//     but want 128 rows of one operand and an 8-bit other one: at most 8 query heads share a page, and rounding
//     queries and weights to 8 bits costs more than the cache's own rounding.)
//   - keys are the M side of both products: S^T[16 keys x 8 heads] = K Q^T, O^T[dims x 8 heads] += V^T P^T, so that up to
//     8 heads fill the N side and no row is wasted.  S^T comes out with keys along the lanes, P^T is wanted with keys
//     along the registers: one 8x8 transpose (movmatrix) per eight keys.
//   - a thread reads 4 consecutive codes of a row as 4 contracted elements (Q is laid out to match), and 16 dimensions of
//     each of 4 keys of V, whose bytes are paired up by two byte permutations per 8 codes.
//   - TMA brings pages with the 128-byte swizzle; the order in which a page's keys take the rows of the MMA is chosen so
//     that both read patterns touch every bank once (key_of_row).
//   - the running maxima are raised only when a score passes them by 2^9: weights have headroom in f16, and the
//     reduction over the lanes and the rescaling of the accumulators are rare.
// Weights carry V's page scale into f16, w_j = 2^(s_j + log2 vs - m_o), with a maximum m_o of their own, so that pages
// whose scales lie far apart neither overflow nor vanish; the denominator keeps the plain maximum m_l.
//
// Work: the (block, kv head, page) triples of all blocks are laid end to end and cut into equal ranges, one per CTA of
// the one wave, from the lengths on the device.  A CTA is one producer warp and four consumer warps around a ring of
// stages; a stage is a round of up to 4 * TP pages of one (block, kv head), with their scales, and with the queries
// (first round) and the new rows (last page) that belong to it: the consumers load nothing from global memory.  Consumer
// w takes pages w, w + 4, ... of a round and keeps its own maxima, sums and O; at the end of a (block, kv head) inside
// the range the four are merged through the stage that they have just consumed.  A range boundary inside a (block, kv
// head) leaves partials in the workspace, and the last CTA to arrive (a counter in the tables) merges them in order.
#include <algorithm>
#include <atomic>

#include "cache_q8.cuh"
#include "cpa_tcgen05.cuh"

namespace {

constexpr int kCons = 4;                              // consumer warps
constexpr int kQ8Threads = (kCons + 1) * 32;
constexpr int kCtasPerSm = 2;
constexpr int kStages = 3;
constexpr uint32_t kQ8Spin = 1u << 18;                // bounded waits (each try suspends briefly)
constexpr float kBase = 6.f, kSlack = 9.f;            // weights: 2^kBase at the maximum, up to 2^(kBase + kSlack) above it

template <int D>
struct Q8Shape {
    static constexpr int TP = D == 128 ? 2 : 4;       // pages per consumer warp and round
    static constexpr int kRound = kCons * TP;         // pages of a round
    static constexpr int kPageBytes = 2 * kPage * D;  // K and V codes of a (page, kv head)
    static constexpr int kData = kRound * kPageBytes;
    // behind a stage's pages: queries, the new K and V rows, scales, the round's descriptor, and (max, sum, max) of the
    // four warps for the merge
    static constexpr int kQ = 0, kNew = kQ + 8 * D * 2, kScale = kNew + 2 * D * 2, kDesc = kScale + kRound * 8,
                         kMl = kDesc + 48, kLast = kMl + kCons * 8 * 16, kMeta = (kLast + 16 + 127) / 128 * 128;
    static constexpr int kSmem = kStages * (kData + kMeta) + 1024;
};

struct round_desc {
    int b, g, page0, n;       // pages [page0, page0 + n) of block b, kv head g; n == 0: the end
    int flags;                // 1: first round of the segment, 2: last, 4: the last page takes the new row
    int len;                  // the block's tokens, the new one included
    int parts, slot;          // CTAs that share the (block, kv head); this one's partial slot
    int slot0, last_slot;     // partial slots: slot0 of the first CTA, then the even ones up to last_slot
    int row;                  // page row of the pages' first code: where the new row goes
    int pad;
};
static_assert(sizeof(round_desc) == 48, "a descriptor is three 16-byte words");

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];\n" : "=r"(r.x), "=r"(r.y) : "r"(a));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float d;
    asm("ex2.approx.f32 %0, %1;\n" : "=f"(d) : "f"(x));
    return d;
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
__device__ __forceinline__ uint32_t f16_lo(uint32_t w) { return e4m3x2_to_f16x2((uint16_t)w); }
__device__ __forceinline__ uint32_t f16_hi(uint32_t w) { return e4m3x2_to_f16x2((uint16_t)(w >> 16)); }

// Byte offset of the 16-byte piece p of token row r inside a swizzled chunk (K or V) of a page.
template <int D>
__device__ __forceinline__ int piece_at(int r, int p) {
    if (D == 128) return r * 128 + ((p ^ (r & 7)) << 4);
    const int line = r >> 1;                          // two rows of 64 codes share a 128-byte line
    return line * 128 + ((((r & 1) * 4 + p) ^ (line & 7)) << 4);
}
// The key (row of the page) that row i of the MMA's M side stands for.  Lane (g, t) reads K rows key(g), key(g + 8) and V
// rows key(2t), key(2t + 1), key(2t + 8), key(2t + 9); with these orders and the swizzle every quarter warp's reads fall
// into eight different 16-byte columns.
template <int D>
__device__ __forceinline__ int key_of_row(int i) {
    if (D == 128) return i ^ ((i & 1) << 2);
    return ((i & 7) >> 1) * 4 + (i & 1) + (i >> 3) * 2;
}

// A block's tokens as this launch sees them, or -1 when it sits out.
__device__ __forceinline__ int block_len(int b, const q8_tables& t, const int32_t* __restrict__ lens,
                                         const int32_t* __restrict__ active, int append, int& ip, int& status) {
    status = 0;
    ip = __ldg(t.page_indptr + b);
    if (active && active[b] == 0) return -1;
    const int64_t room = (int64_t)(__ldg(t.page_indptr + b + 1) - ip) * kPage, len = lens[b];
    if (len < 0) status = kStatusInvalid;
    else if (len + append > room) status = kStatusNoSpace;
    return status ? -1 : (int)len + append;
}

struct q8_args {
    q8_tables t;
    const __nv_bfloat16 *q, *k_new, *v_new;
    const int32_t* lens;
    int32_t* lens_out;
    const int32_t* active;
    uint8_t* pool;
    float* scales;
    __nv_bfloat16* o;
    float* ws;                 // [slots, G, D] accumulators, then [slots, G, 4] (max, sum, max of the weights, -)
    int B, Hq, Hkv, G;
    float scale_log2;
    int min_quota;             // pages of a CTA's range at least
};

// Stores a finished row pair: dims d, d + 1 of query head h.
__device__ __forceinline__ void store_pair(const q8_args& a, int b, int g, int h, int D, int d, float o0, float o1, float L,
                                           float Mo, float Ml) {
    // the factor 2^(Mo - kBase - Ml) in two halves: on its own it may leave fp32's range where the result does not
    const float e = ex2(0.5f * (Mo - kBase - Ml)), inv = 1.f / L;
    *reinterpret_cast<__nv_bfloat162*>(a.o + ((int64_t)b * a.Hq + g * a.G + h) * D + d) =
        __floats2bfloat162_rn(o0 * inv * e * e, o1 * inv * e * e);
}

template <int D>
__global__ void __launch_bounds__(kQ8Threads, kCtasPerSm)
decode_q8_kernel(const __grid_constant__ CUtensorMap tm, const q8_args a) {
    using Sh = Q8Shape<D>;
    constexpr int TP = Sh::TP;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t sm_full[kStages], sm_empty[kStages], sm_flush;
    __shared__ int sm_scan[kQ8Threads / 32], sm_start[3];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t data0 = (smem_u32(raw) + 1023u) & ~1023u, meta0 = data0 + kStages * Sh::kData;
    const uint32_t full0 = smem_u32(sm_full), empty0 = smem_u32(sm_empty), flush_bar = smem_u32(&sm_flush);
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, kCons); }
        mbar_init(flush_bar, kCons * 32);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
        sm_start[0] = a.B;
    }
    // everything above touches nothing that an earlier launch writes; this one may have been started before that one ended
    asm volatile("griddepcontrol.wait;\n" ::: "memory");

    // ---- the cut: every thread takes a run of blocks, and the runs' page counts are scanned
    const int append = a.k_new != nullptr;
    const int run = (a.B + kQ8Threads - 1) / kQ8Threads, b_lo = min(a.B, tid * run), b_hi = min(a.B, b_lo + run);
    int mine = 0;
    for (int b = b_lo; b < b_hi; ++b) {
        int ip, status;
        const int len = block_len(b, a.t, a.lens, a.active, append, ip, status);
        if (len > 0) mine += (len + kPage - 1) / kPage;
        if (b % (int)gridDim.x != (int)blockIdx.x) continue;
        // this CTA keeps block b's books: status, new length, and the zero row of an empty block
        if (status) atomicCAS(a.t.header, 0, status);
        if (a.lens_out) a.lens_out[b] = len < 0 ? a.lens[b] : len;
        if (len == 0)
            for (int i = 0; i < a.Hq * (D / 8); ++i)
                reinterpret_cast<uint4*>(a.o + (int64_t)b * a.Hq * D)[i] = make_uint4(0, 0, 0, 0);
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += v;
    }
    if (lane == 31) sm_scan[warp] = inc;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kQ8Threads / 32; ++w) {
        if (w < warp) before += sm_scan[w];
        total += sm_scan[w];
    }
    before += inc - mine;
    const int64_t all = (int64_t)total * a.Hkv;
    const int64_t quota = max((all + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)a.min_quota);
    const int64_t x0 = quota * blockIdx.x, x1 = min(x0 + quota, all);
    if (x0 >= x1) return;                              // (uniform) more CTAs than work
    if (mine > 0 && x0 >= (int64_t)before * a.Hkv && x0 < (int64_t)(before + mine) * a.Hkv) {
        int64_t x = (int64_t)before * a.Hkv;
        for (int b = b_lo; b < b_hi; ++b) {            // the block that the range starts in, and where in it
            int ip, status;
            const int len = block_len(b, a.t, a.lens, a.active, append, ip, status);
            const int64_t units = len > 0 ? (int64_t)((len + kPage - 1) / kPage) * a.Hkv : 0;
            if (x0 < x + units) {
                sm_start[0] = b;
                sm_start[1] = (int)((x0 - x) / (units / a.Hkv));
                sm_start[2] = (int)((x0 - x) % (units / a.Hkv));
                break;
            }
            x += units;
        }
    }
    __syncthreads();

    bool dead = false;
    if (warp == kCons) {
        // ================================================================ producer
        // A window of 32 blocks in the lanes' registers: tokens and first entry of the page list.
        int win = sm_start[0], w_len, w_ip;
        auto window = [&]() {
            int status;
            w_len = -1;
            w_ip = 0;
            if (win + lane < a.B) w_len = block_len(win + lane, a.t, a.lens, a.active, append, w_ip, status);
        };
        window();
        int b = sm_start[0], g = sm_start[1], p = sm_start[2];
        int64_t left = x1 - x0, unit0 = x0 - p;         // pages of the range still to hand out; where this unit starts
        int len = __shfl_sync(0xffffffffu, w_len, 0), ip = __shfl_sync(0xffffffffu, w_ip, 0);
        int pages = (len + kPage - 1) / kPage;
        bool opened = false;                            // a round of this unit has been handed out
        // the next round of the range into `r`; its page list entries start at `ids`
        auto next = [&](round_desc& r, int& ids) {
            r.n = 0;
            if (left <= 0) return;
            if (p == pages) {                           // on to the next kv head, or the next block that has pages
                unit0 += pages;
                p = 0;
                opened = false;
                if (++g == a.Hkv) {
                    g = 0;
                    do {
                        if (++b >= win + 32) { win = b; window(); }
                        len = __shfl_sync(0xffffffffu, w_len, b - win);
                    } while (len <= 0 && b < a.B);
                    if (b >= a.B) { left = 0; return; }  // (cannot be reached: the range ends inside the blocks)
                    ip = __shfl_sync(0xffffffffu, w_ip, b - win);
                    pages = (len + kPage - 1) / kPage;
                }
            }
            r.b = b;
            r.g = g;
            r.page0 = p;
            r.n = (int)min((int64_t)min(pages - p, Sh::kRound), left);
            r.len = len;
            ids = ip + p;
            p += r.n;
            left -= r.n;
            r.flags = (opened ? 0 : 1) | (p == pages || left == 0 ? 2 : 0) | (append && p == pages ? 4 : 0);
            opened = true;
            const int64_t c0 = unit0 / quota, c1 = (unit0 + pages - 1) / quota;
            r.parts = (int)(c1 - c0) + 1;
            r.slot0 = (int)(2 * c0 + 1);
            r.last_slot = (int)(2 * c1);
            r.slot = (int)blockIdx.x == (int)c0 ? r.slot0 : 2 * (int)blockIdx.x;
            r.pad = 0;
        };
        // three rounds in flight: descriptor and page ids two ahead, scales one ahead
        round_desc d0, d1, d2;
        int at = 0, id0 = 0, id1 = 0, id2 = 0;
        float2 sc0 = make_float2(0.f, 0.f), sc1 = sc0;
        next(d0, at);
        if (lane < d0.n) id0 = __ldg(a.t.page_indices + at + lane);
        next(d1, at);
        if (lane < d1.n) id1 = __ldg(a.t.page_indices + at + lane);
        // (scales are read past the caches that __ldg may use: the append writes them in this launch)
        if (lane < d0.n) sc0 = __ldcg(reinterpret_cast<const float2*>(a.scales) + (int64_t)id0 * a.Hkv + d0.g);
        int it = 0;
        for (;; ++it) {
            next(d2, at);
            id2 = 0;
            if (lane < d2.n) id2 = __ldg(a.t.page_indices + at + lane);
            if (lane < d1.n) sc1 = __ldcg(reinterpret_cast<const float2*>(a.scales) + (int64_t)id1 * a.Hkv + d1.g);
            const int st = it % kStages;
            if (it >= kStages) mbar_wait(empty0 + 8 * st, (uint32_t)(it / kStages - 1) & 1u, dead, a.t.header, kQ8Spin);
            if (__any_sync(0xffffffffu, dead)) break;
            const uint32_t data = data0 + st * Sh::kData, meta = meta0 + st * Sh::kMeta, bar = full0 + 8 * st;
            d0.row = (id0 * a.Hkv + d0.g);
            d0.row = __shfl_sync(0xffffffffu, d0.row, d0.n > 0 ? d0.n - 1 : 0);    // (page, head) of the round's last page
            if (lane < d0.n) {
                asm volatile("st.shared.v2.f32 [%0], {%1,%2};\n" :: "r"(meta + Sh::kScale + 8 * lane), "f"(sc0.x), "f"(sc0.y) : "memory");
            }
            if (lane == 0) {
                const int4* w = reinterpret_cast<const int4*>(&d0);
                for (int i = 0; i < 3; ++i)
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};\n"
                                 :: "r"(meta + Sh::kDesc + 16 * i), "r"(w[i].x), "r"(w[i].y), "r"(w[i].z), "r"(w[i].w) : "memory");
            }
            __syncwarp();
            if (d0.n == 0) {                            // the end: no copies, the stage is complete at once
                if (lane == 0) mbar_arrive(bar);
                break;
            }
            if (lane == 0) {
                mbar_expect_tx(bar, d0.n * Sh::kPageBytes + (d0.flags & 1 ? a.G * D * 2 : 0) + (d0.flags & 4 ? 2 * D * 2 : 0));
                if (d0.flags & 1) bulk_copy(meta + Sh::kQ, a.q + ((int64_t)d0.b * a.Hq + d0.g * a.G) * D, a.G * D * 2, bar);
                if (d0.flags & 4) {
                    const int64_t row = ((int64_t)d0.b * a.Hkv + d0.g) * D;
                    bulk_copy(meta + Sh::kNew, a.k_new + row, D * 2, bar);
                    bulk_copy(meta + Sh::kNew + D * 2, a.v_new + row, D * 2, bar);
                }
            }
            __syncwarp();
            if (lane < d0.n) tma_load_2d(data + lane * Sh::kPageBytes, &tm, 0, (id0 * a.Hkv + d0.g) * (Sh::kPageBytes / 128), bar);
            d0 = d1;
            d1 = d2;
            id0 = id1;
            id1 = id2;
            sc0 = sc1;
        }
        if (__any_sync(0xffffffffu, dead)) {            // a wait gave up: see the copies in flight through before leaving
            if (lane == 0)
                for (int i = max(0, it - kStages); i < it; ++i)
                    mbar_drain(full0 + 8 * (i % kStages), (uint32_t)(i / kStages) & 1u, kDrainLimit);
            __syncwarp();
        }
        return;
    }

    // ==================================================================== consumers
    const int g8 = lane >> 2, t4 = lane & 3;
    uint32_t flush_phase = 0;
    auto flush_wait = [&]() {                           // all consumer threads, bounded
        mbar_arrive(flush_bar);
        mbar_wait(flush_bar, flush_phase, dead, a.t.header, kQ8Spin);
        flush_phase ^= 1u;
        dead = __any_sync(0xffffffffu, dead);
    };
    uint32_t qf[D / 64][4][2];
    float acc[D / 16][4], c0 = 0.f, c1 = 0.f;           // c: what a score's sum is multiplied with, for heads 2t, 2t + 1
    float ml0 = -INFINITY, ml1 = -INFINITY, mo0 = -INFINITY, mo1 = -INFINITY, l0 = 0.f, l1 = 0.f;

    for (int it = 0;; ++it) {
        const int st = it % kStages;
        const uint32_t data = data0 + st * Sh::kData, meta = meta0 + st * Sh::kMeta;
        mbar_wait(full0 + 8 * st, (uint32_t)(it / kStages) & 1u, dead, a.t.header, kQ8Spin);
        if (__any_sync(0xffffffffu, dead)) return;
        const uint4 e0 = lds16(meta + Sh::kDesc), e1 = lds16(meta + Sh::kDesc + 16);
        const int page0 = (int)e0.z, n = (int)e0.w, flags = (int)e1.x, len = (int)e1.y;
        if (n == 0) return;
        if (flags & 1) {
            // the queries as f16 B fragments: contracted elements 2t, 2t+1, 2t+8, 2t+9 of step (p, w) are dimensions
            // 64 p + 16 t + 4 w + 0 .. 3.  2^7 at the row's largest element.
            uint4 v[D / 64][2];
            uint32_t amax = 0;
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    v[p][i] = g8 < a.G ? lds16(meta + Sh::kQ + (g8 * D + 64 * p + 16 * t4 + 8 * i) * 2) : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {v[p][i].x, v[p][i].y, v[p][i].z, v[p][i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) amax = max(amax, max((w[j] << 16) & 0x7FFFFFFFu, w[j] & 0x7FFF0000u));
                }
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            int e = (int)(amax >> 23);                   // biased exponent; infinities and NaN go through as they are
            e = amax == 0 || e == 255 ? 134 : max(e, 8);
            const float up = __uint_as_float((uint32_t)(261 - e) << 23), down = __uint_as_float((uint32_t)(e - 7) << 23);
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w[4] = {v[p][i].x, v[p][i].y, v[p][i].z, v[p][i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        qf[p][2 * i + (j >> 1)][j & 1] = pack_f16(__uint_as_float(w[j] << 16) * up, __uint_as_float(w[j] & 0xFFFF0000u) * up);
                }
            const float c = down * a.scale_log2;
            c0 = __shfl_sync(0xffffffffu, c, 8 * t4);
            c1 = __shfl_sync(0xffffffffu, c, 8 * t4 + 4);
            ml0 = ml1 = mo0 = mo1 = -INFINITY;
            l0 = l1 = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
        }
        const int n_mine = (n - warp + kCons - 1) / kCons;   // this warp's pages of the round (may be 0)

        if ((flags & 4) && n_mine > 0 && warp + kCons * (n_mine - 1) == n - 1) {
            // ---- the block's newest page is this warp's: quantise the new row into it, here and in the pool
            const int slot = (len - 1) % kPage, j = n - 1;
            const uint32_t chunk0 = data + j * Sh::kPageBytes;
            const int64_t cell = (int64_t)(int)lds16(meta + Sh::kDesc + 32).z;       // page * Hkv + g
#pragma unroll
            for (int kind = 0; kind < 2; ++kind) {
                const uint32_t chunk = chunk0 + kind * (kPage * D);
                uint8_t* to = a.pool + cell * Sh::kPageBytes + kind * (kPage * D);
                float x[D / 32];                             // dimensions lane * D / 32 ..
                uint32_t amax = 0;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    uint32_t w;
                    asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(w) : "r"(meta + Sh::kNew + kind * D * 2 + (lane * (D / 64) + i) * 4));
                    x[2 * i] = __uint_as_float(w << 16);
                    x[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
                    amax = max(amax, max(q8_finite_abs(w << 16), q8_finite_abs(w & 0xFFFF0000u)));
                }
                amax = __reduce_max_sync(0xffffffffu, amax);
                float s = q8_scale(amax);
                const uint32_t sc_at = meta + Sh::kScale + 8 * j + 4 * kind;
                if (slot > 0) {
                    float old;
                    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(old) : "r"(sc_at));
                    if (s > old) {
                        const float f = old * q8_inverse(s);
                        for (int i = lane; i < slot * (D / 4); i += 32) {
                            const int r = i / (D / 4), c = i % (D / 4);
                            const uint32_t at = chunk + piece_at<D>(r, c >> 2) + (c & 3) * 4;
                            uint32_t w;
                            asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(w) : "r"(at));
                            w = q8_rescale4(w, f);
                            asm volatile("st.shared.u32 [%0], %1;\n" :: "r"(at), "r"(w) : "memory");
                            reinterpret_cast<uint32_t*>(to)[i] = w;
                        }
                    } else {
                        s = old;
                    }
                }
                const bool pow2 = (__float_as_uint(s) & 0x807FFFFFu) == 0 && s <= 0x1p120f;
                const float inv = pow2 ? q8_inverse(s) : 1.f / s;
                uint32_t codes = to_e4m3x2(mul_keep(x[0], inv), mul_keep(x[1], inv));
                if (D == 128) codes |= to_e4m3x2(mul_keep(x[D / 32 - 2], inv), mul_keep(x[D / 32 - 1], inv)) << 16;
                const int byte = lane * (D / 32);
                const uint32_t at = chunk + piece_at<D>(slot, byte >> 4) + (byte & 15);
                if (D == 128) {
                    asm volatile("st.shared.u32 [%0], %1;\n" :: "r"(at), "r"(codes) : "memory");
                    *reinterpret_cast<uint32_t*>(to + slot * D + byte) = codes;
                } else {
                    asm volatile("st.shared.u16 [%0], %1;\n" :: "r"(at), "h"((uint16_t)codes) : "memory");
                    *reinterpret_cast<uint16_t*>(to + slot * D + byte) = (uint16_t)codes;
                }
                __syncwarp();                                // every lane has read the old scale
                if (lane == 0) {
                    asm volatile("st.shared.f32 [%0], %1;\n" :: "r"(sc_at), "f"(s) : "memory");
                    a.scales[cell * 2 + kind] = s;
                }
            }
            fence_async();                                   // the copy that refills the stage comes after these stores
            __syncwarp();
        }

        // ---- scores of this warp's pages: s[i] = (key(g), head 2t), (key(g), 2t+1), (key(g+8), 2t), (key(g+8), 2t+1)
        float s[TP][4], lv[TP];
        float hi0 = -INFINITY, hi1 = -INFINITY, ho0 = -INFINITY, ho1 = -INFINITY;
#pragma unroll
        for (int i = 0; i < TP; ++i) {
            if (i >= n_mine) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][e] = -INFINITY;
                lv[i] = 0.f;
                continue;
            }
            const int j = warp + kCons * i;
            const uint32_t kc = data + j * Sh::kPageBytes;
            const uint2 sc = lds8(meta + Sh::kScale + 8 * j);
            float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < D / 64; ++p) {
                const uint4 r0 = lds16(kc + piece_at<D>(key_of_row<D>(g8), t4 + 4 * p));
                const uint4 r1 = lds16(kc + piece_at<D>(key_of_row<D>(g8 + 8), t4 + 4 * p));
                mma_f16(sa, f16_lo(r0.x), f16_lo(r1.x), f16_hi(r0.x), f16_hi(r1.x), qf[p][0][0], qf[p][0][1]);
                mma_f16(sb, f16_lo(r0.y), f16_lo(r1.y), f16_hi(r0.y), f16_hi(r1.y), qf[p][1][0], qf[p][1][1]);
                mma_f16(sa, f16_lo(r0.z), f16_lo(r1.z), f16_hi(r0.z), f16_hi(r1.z), qf[p][2][0], qf[p][2][1]);
                mma_f16(sb, f16_lo(r0.w), f16_lo(r1.w), f16_hi(r0.w), f16_hi(r1.w), qf[p][3][0], qf[p][3][1]);
            }
            const float ks = __uint_as_float(sc.x), k0 = ks * c0, k1 = ks * c1;
            s[i][0] = (sa[0] + sb[0]) * k0;
            s[i][1] = (sa[1] + sb[1]) * k1;
            s[i][2] = (sa[2] + sb[2]) * k0;
            s[i][3] = (sa[3] + sb[3]) * k1;
            asm("lg2.approx.f32 %0, %1;\n" : "=f"(lv[i]) : "f"(__uint_as_float(sc.y)));
            const int valid = len - (page0 + j) * kPage;     // slots behind it may hold anything
            if (valid < kPage) {
                if (key_of_row<D>(g8) >= valid) s[i][0] = s[i][1] = -INFINITY;
                if (key_of_row<D>(g8 + 8) >= valid) s[i][2] = s[i][3] = -INFINITY;
            }
            const float a0 = fmaxf(s[i][0], s[i][2]), a1 = fmaxf(s[i][1], s[i][3]);
            hi0 = fmaxf(hi0, a0);
            hi1 = fmaxf(hi1, a1);
            ho0 = fmaxf(ho0, a0 + lv[i]);
            ho1 = fmaxf(ho1, a1 + lv[i]);
        }
        if (n_mine > 0) {
            // ---- raise the maxima when a score has passed them by more than the headroom (always at the first page)
            const bool passed = hi0 > ml0 + kSlack || hi1 > ml1 + kSlack || ho0 > mo0 + kSlack || ho1 > mo1 + kSlack;
            if (__any_sync(0xffffffffu, passed)) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    hi0 = fmaxf(hi0, __shfl_xor_sync(0xffffffffu, hi0, o));
                    hi1 = fmaxf(hi1, __shfl_xor_sync(0xffffffffu, hi1, o));
                    ho0 = fmaxf(ho0, __shfl_xor_sync(0xffffffffu, ho0, o));
                    ho1 = fmaxf(ho1, __shfl_xor_sync(0xffffffffu, ho1, o));
                }
                auto raise = [](float& m, float hi) {        // the factor of what was summed under the old maximum
                    const float up = fmaxf(m, hi), f = m == -INFINITY ? 0.f : ex2(m - up);
                    m = up;
                    return f;
                };
                l0 *= raise(ml0, hi0);
                l1 *= raise(ml1, hi1);
                const float f0 = raise(mo0, ho0), f1 = raise(mo1, ho1);
#pragma unroll
                for (int j = 0; j < D / 16; ++j) { acc[j][0] *= f0; acc[j][1] *= f1; acc[j][2] *= f0; acc[j][3] *= f1; }
            }
            // ---- weights, and O^T += V^T P^T
            const float b0 = kBase - mo0, b1 = kBase - mo1;
#pragma unroll
            for (int i = 0; i < TP; ++i) {
                if (i >= n_mine) continue;
                const int j = warp + kCons * i;
                l0 += ex2(s[i][0] - ml0) + ex2(s[i][2] - ml0);
                l1 += ex2(s[i][1] - ml1) + ex2(s[i][3] - ml1);
                const float u0 = b0 + lv[i], u1 = b1 + lv[i];
                const uint32_t p0 = transpose8(pack_f16(ex2(s[i][0] + u0), ex2(s[i][1] + u1)));
                const uint32_t p1 = transpose8(pack_f16(ex2(s[i][2] + u0), ex2(s[i][3] + u1)));
                const uint32_t vc = data + j * Sh::kPageBytes + kPage * D;
                const int valid = len - (page0 + j) * kPage;
                constexpr int W = D / 32;                    // words of codes per lane and key
                uint32_t v[4][W];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = key_of_row<D>(2 * t4 + (r & 1) + 8 * (r >> 1));
                    if (D == 128) {
                        const uint4 x = lds16(vc + piece_at<D>(key, g8));
                        v[r][0] = x.x; v[r][1] = x.y; v[r][W - 2] = x.z; v[r][W - 1] = x.w;
                    } else {
                        const uint2 x = lds8(vc + piece_at<D>(key, g8 >> 1) + (g8 & 1) * 8);
                        v[r][0] = x.x; v[r][1] = x.y;
                    }
                    if (valid < kPage && key >= valid) {     // a weight of zero would not silence a NaN
#pragma unroll
                        for (int w = 0; w < W; ++w) v[r][w] = 0u;
                    }
                }
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    // codes of two keys side by side: (dims 0, 1 of the word) and (dims 2, 3)
                    const uint32_t a01 = __byte_perm(v[0][w], v[1][w], 0x5140), a23 = __byte_perm(v[0][w], v[1][w], 0x7362);
                    const uint32_t b01 = __byte_perm(v[2][w], v[3][w], 0x5140), b23 = __byte_perm(v[2][w], v[3][w], 0x7362);
                    mma_f16(acc[2 * w], f16_lo(a01), f16_hi(a01), f16_lo(b01), f16_hi(b01), p0, p1);
                    mma_f16(acc[2 * w + 1], f16_lo(a23), f16_hi(a23), f16_lo(b23), f16_hi(b23), p0, p1);
                }
            }
        }
        __syncwarp();
        if (!(flags & 2)) {
            if (lane == 0) mbar_arrive(empty0 + 8 * st);
            continue;
        }

        // ---- the segment is done: merge the four warps through the stage (each writes over its own first page)
        l0 += __shfl_xor_sync(0xffffffffu, l0, 4);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 4);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 8);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 8);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 16);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 16);
        // row h of [8][D] floats, as pairs: pair u sits at u ^ swz(u, h), so that neither side meets a bank twice
        auto pair_at = [](int h, int u) {
            const int x = D == 128 ? ((u >> 4) & 1) << 2 : 0;
            return (h * (D / 2) + (u ^ x ^ (h >> 1))) * 8;
        };
        const uint32_t mine_o = data + warp * Sh::kPageBytes;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const int u = g8 * (D / 16) + j;                 // dims 2u, 2u + 1 = rows g, g + 8 of tile j
            asm volatile("st.shared.v2.f32 [%0], {%1,%2};\n" :: "r"(mine_o + pair_at(2 * t4, u)), "f"(acc[j][0]), "f"(acc[j][2]) : "memory");
            asm volatile("st.shared.v2.f32 [%0], {%1,%2};\n" :: "r"(mine_o + pair_at(2 * t4 + 1, u)), "f"(acc[j][1]), "f"(acc[j][3]) : "memory");
        }
        if (g8 == 0) {
            const uint32_t to = meta + Sh::kMl + (warp * 8 + 2 * t4) * 16;
            asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%3};\n" :: "r"(to), "f"(ml0), "f"(l0), "f"(mo0) : "memory");
            asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%3};\n" :: "r"(to + 16), "f"(ml1), "f"(l1), "f"(mo1) : "memory");
        }
        fence_async();
        flush_wait();
        if (dead) return;
        const int blk = (int)e0.x, head = (int)e0.y;
        const uint4 e2 = lds16(meta + Sh::kDesc + 32);
        const int parts = (int)e1.z, slot = (int)e1.w, slot0 = (int)e2.x, last_slot = (int)e2.y;
        float* ws_o = a.ws;
        float4* ws_ml = reinterpret_cast<float4*>(a.ws + (int64_t)2 * gridDim.x * a.G * D);
        for (int i = tid; i < a.G * (D / 2); i += kCons * 32) {
            const int h = i / (D / 2), u = i % (D / 2);
            float4 m[kCons];
            float Ml = -INFINITY, Mo = -INFINITY, L = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
            for (int w = 0; w < kCons; ++w) {
                const uint4 x = lds16(meta + Sh::kMl + (w * 8 + h) * 16);
                m[w] = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), 0.f);
                Ml = fmaxf(Ml, m[w].x);
                Mo = fmaxf(Mo, m[w].z);
            }
#pragma unroll
            for (int w = 0; w < kCons; ++w) {
                const uint2 x = lds8(data + w * Sh::kPageBytes + pair_at(h, u));
                const float f = m[w].z == -INFINITY ? 0.f : ex2(m[w].z - Mo);
                // (a warp that had no page holds zeros under a maximum of -inf)
                L += m[w].x == -INFINITY ? m[w].y : ex2(m[w].x - Ml) * m[w].y;
                o0 = fmaf(f, __uint_as_float(x.x), o0);
                o1 = fmaf(f, __uint_as_float(x.y), o1);
            }
            if (parts == 1) {
                store_pair(a, blk, head, h, D, 2 * u, o0, o1, L, Mo, Ml);
            } else {
                const int64_t row = (int64_t)slot * a.G + h;
                *reinterpret_cast<float2*>(ws_o + row * D + 2 * u) = make_float2(o0, o1);
                if (u == 0) ws_ml[row] = make_float4(Ml, L, Mo, 0.f);
            }
        }
        if (parts > 1) {
            // ---- the last of the CTAs that share this (block, kv head) merges their partials, in order
            __threadfence();
            flush_wait();
            if (dead) return;
            if (tid == 0) {
                __threadfence();
                const unsigned before_me = atomicInc(reinterpret_cast<unsigned*>(a.t.tickets) + (int64_t)blk * a.Hkv + head,
                                                     (unsigned)parts - 1);           // back to zero with the last one
                asm volatile("st.shared.u32 [%0], %1;\n" :: "r"(meta + Sh::kLast), "r"(before_me == (unsigned)parts - 1 ? 1u : 0u) : "memory");
            }
            flush_wait();
            if (dead) return;
            uint32_t last;
            asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(last) : "r"(meta + Sh::kLast));
            if (last) {
                __threadfence();
                auto slot_of = [&](int i) { return i == 0 ? slot0 : slot0 + 2 * i - 1; };
                (void)last_slot;
                for (int i = tid; i < a.G * (D / 2); i += kCons * 32) {
                    const int h = i / (D / 2), u = i % (D / 2);
                    float Ml = -INFINITY, Mo = -INFINITY, L = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll 4
                    for (int k = 0; k < parts; ++k) {
                        const float4 m = __ldcg(ws_ml + (int64_t)slot_of(k) * a.G + h);
                        Ml = fmaxf(Ml, m.x);
                        Mo = fmaxf(Mo, m.z);
                    }
#pragma unroll 4
                    for (int k = 0; k < parts; ++k) {
                        const int64_t row = (int64_t)slot_of(k) * a.G + h;
                        const float4 m = __ldcg(ws_ml + row);
                        const float2 x = __ldcg(reinterpret_cast<const float2*>(ws_o + row * D + 2 * u));
                        const float f = ex2(m.z - Mo);
                        L = fmaf(ex2(m.x - Ml), m.y, L);
                        o0 = fmaf(f, x.x, o0);
                        o1 = fmaf(f, x.y, o1);
                    }
                    store_pair(a, blk, head, h, D, 2 * u, o0, o1, L, Mo, Ml);
                }
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * st);
    }
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// SMs of the current device, 0 if there is none (asked once per device).
int device_sms(int dev) {
    static std::atomic<int> known[64];
    int n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
            (void)cudaGetLastError();
            return 0;
        }
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

constexpr int kSmsByDefault = 148;                     // what the workspace is sized for when num_sms is 0

template <int D>
int launch_q8(const cpa_config* cfg, const cpa_table_dims* dims, q8_args& a, cudaStream_t st) {
    using Sh = Q8Shape<D>;
    static std::atomic<bool> configured[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { (void)cudaGetLastError(); return CPA_ECUDA; }
    if (!configured[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(decode_q8_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return CPA_ECUDA;
        }
        configured[dev].store(true, std::memory_order_relaxed);
    }
    const int sms = cfg->num_sms ? cfg->num_sms : std::min(device_sms(dev), kSmsByDefault);
    if (sms <= 0) return CPA_ECUDA;
    // The pool as lines of 128 bytes; a box is the K and V codes of one (page, kv head).
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return CPA_ECUDA;
    CUtensorMap tm;
    const cuuint64_t size[2] = {128, (cuuint64_t)dims->num_pages * cfg->num_kv_heads * (Sh::kPageBytes / 128)};
    const cuuint64_t stride[1] = {128};
    const cuuint32_t box[2] = {128, Sh::kPageBytes / 128}, elem[2] = {1, 1};
    if (fn(&tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, a.pool, size, stride, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return CPA_ECUDA;
    a.min_quota = Sh::kRound;
    // one wave; no more CTAs than the table's pages could keep busy, or the blocks' books need
    const int64_t most = ((int64_t)dims->page_capacity * cfg->num_kv_heads + a.min_quota - 1) / a.min_quota;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(kCtasPerSm * sms, most)));
    lc.blockDim = dim3(kQ8Threads);
    lc.dynamicSmemBytes = Sh::kSmem;
    lc.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    if (cudaLaunchKernelEx(&lc, decode_q8_kernel<D>, tm, a) != cudaSuccess) { (void)cudaGetLastError(); return CPA_ECUDA; }
    return CPA_OK;
}

int decode(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* q, const void* k_new,
           const void* v_new, const int32_t* d_lens, int32_t* d_lens_out, const int32_t* d_active, void* kv_pool,
           float* kv_scales, void* o, void* d_workspace, void* stream) {
    const int rc = q8_check(cfg, dims);
    if (rc != CPA_OK) return rc;
    if (!d_tables || !q || !d_lens || !kv_pool || !kv_scales || !o || !d_workspace || !cpa_aligned16(d_tables) ||
        !cpa_aligned16(q) || !cpa_aligned16(kv_pool) || !cpa_aligned16(kv_scales) || !cpa_aligned16(o) ||
        !cpa_aligned16(d_workspace) || !aligned4(d_lens) || !aligned4(d_lens_out) || !aligned4(d_active))
        return CPA_EINVAL;
    q8_args a{q8_view(*cfg, *dims, d_tables), (const __nv_bfloat16*)q, (const __nv_bfloat16*)k_new,
              (const __nv_bfloat16*)v_new, d_lens, d_lens_out, d_active, (uint8_t*)kv_pool, kv_scales, (__nv_bfloat16*)o,
              (float*)d_workspace, dims->num_blocks, cfg->num_q_heads, cfg->num_kv_heads,
              cfg->num_q_heads / cfg->num_kv_heads, cfg->scale * 1.4426950408889634f, 0};
    return cfg->head_dim == 128 ? launch_q8<128>(cfg, dims, a, (cudaStream_t)stream)
                                : launch_q8<64>(cfg, dims, a, (cudaStream_t)stream);
}

}  // namespace

extern "C" int64_t cpa_decode_q8_workspace_bytes(const cpa_config* cfg) {
    const cpa_table_dims one{1, 0, 1, 1, 0};
    const int rc = q8_check(cfg, &one);
    if (rc != CPA_OK) return rc;
    // two partial slots per CTA of the wave
    const int64_t slots = 2 * kCtasPerSm * (cfg->num_sms ? cfg->num_sms : kSmsByDefault);
    return slots * (cfg->num_q_heads / cfg->num_kv_heads) * (cfg->head_dim + 4) * 4;
}

extern "C" int cpa_decode_q8(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* q,
                             const int32_t* d_lens, const int32_t* d_active, const void* kv_pool, const float* kv_scales,
                             void* o, void* d_workspace, void* stream) {
    return decode(cfg, dims, d_tables, q, nullptr, nullptr, d_lens, nullptr, d_active, const_cast<void*>(kv_pool),
                  const_cast<float*>(kv_scales), o, d_workspace, stream);
}

extern "C" int cpa_decode_append_q8(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* q,
                                    const void* k_new, const void* v_new, const int32_t* d_lens, int32_t* d_lens_out,
                                    const int32_t* d_active, void* kv_pool, float* kv_scales, void* o, void* d_workspace,
                                    void* stream) {
    if (!k_new || !v_new || !d_lens_out || d_lens == d_lens_out || !cpa_aligned16(k_new) || !cpa_aligned16(v_new))
        return CPA_EINVAL;
    return decode(cfg, dims, d_tables, q, k_new, v_new, d_lens, d_lens_out, d_active, kv_pool, kv_scales, o, d_workspace,
                  stream);
}
