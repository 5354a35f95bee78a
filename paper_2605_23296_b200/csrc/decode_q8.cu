// Decode over the 8-bit cache: one query token per block over that block's pages, with the step's append fused in.
//
//   O[h] = sum_j p_j v_j / sum_j p_j,   p_j = 2^(s_j - m),   s_j = scale log2(e) q[h].k_j,   k, v = code * page scale
//
// The step reads every code once (2 bytes per token, kv head and dimension) and is bound by HBM.  Per SM that is a page
// of one kv head (16 tokens, 4 KB at head_dim 128) every 90 ns, so the arithmetic per page has to stay below that:
//   - codes go to the warp-level MMA (m16n8k16, f16 in, fp32 sums) as f16, which holds an e4m3 value exactly; the page
//     scale of K multiplies the finished score.  The queries are made f16 by a power of two per head, exactly but for
//     elements below 2^-22 of the row's largest, which are off by 2^-32 of it at most.  (The tensor cores of the fifth
//     generation would take the codes as they are, with the keys of eight pages as their 128 rows, a query as the sum of
//     two 8-bit parts and a weight of 11 bits as that of three.  Not built: the stream of pages already runs at the
//     memory's rate, and what is left over it, start and join, is not in the products.)
//   - keys are the M side of both products: S^T[16 keys x 8 heads] = K Q^T, O^T[dims x 8 heads] += V^T P^T, so that up to
//     8 heads fill the N side and no row is wasted.  S^T comes out with keys along the lanes, P^T is wanted with keys
//     along the registers: one 8x8 transpose (movmatrix) per eight keys.
//   - a thread reads 4 consecutive codes of a row as 4 contracted elements (Q is laid out to match), and 16 dimensions of
//     each of 4 keys of V, whose bytes are paired up by two byte permutations per 8 codes.
//   - TMA brings pages with the 128-byte swizzle; the order in which a page's keys take the rows of the MMA is chosen so
//     that both read patterns touch every bank once (key_of_row).
//   - the running maxima are raised only when a score passes them by 2^9: weights have headroom in f16, and the
//     reduction over the lanes and the rescaling of the accumulators are rare.
// Weights carry V's page scale into f16, w_j = 2^(6 + s_j + log2 vs - m_o), with a maximum m_o of their own, so that large
// scales do not overflow and what small ones lose is small beside what large ones add: a weight below 2^-20 of the largest
// loses bits, one below 2^-31 is zero, 2^-31 of the largest is the most that any is off.  (A dimension in which all that
// is large holds zeros shows it.  Weights in more bits would want a product and an accumulation per page: by count 60
// instructions on top of 270, and 32 registers that are not there; not built.)  The denominator keeps the plain maximum
// m_l, in fp32.
//
// Work: the (block, kv head, page) triples of all blocks are laid end to end and cut into ranges from the lengths on the
// device: one equal range per CTA of the one wave.  (Handing the last sixth out in small ranges as CTAs finish was slower,
// 116 us for 63: a range costs its producer a search and its merger a join.)  A CTA is four consumer warps, a producer and
// a merger around a ring of stages; a stage is a round of up to 4 * TP pages of one (block, kv head), with their scales,
// and with the queries (first round) and the new rows (last page) that belong to it: the consumers
// load nothing from global memory.  Consumer w takes pages w, w + 4, ... of a round and keeps its own maxima, sums and
// O; at the end of a (block, kv head) inside a range it leaves them in the stage that it has just consumed and goes on.
// The merger joins the four from there.  A range boundary inside a (block, kv head) leaves partials in the workspace,
// and the merger that arrives last (a counter in the tables) joins them in the order of the ranges.
//
// Measured (one wave of 2 x 148 CTAs): 32 blocks of 1024 .. 8192 tokens, 32 heads over 8 of 128, 337 MB: 60 us, of which
// the stream 48 us (7.0 TB/s) and start and merge the rest; one block of 131072: 50 us; 192 blocks of 512 .. 1024 with
// their append: 58 us; 16 blocks of 8192, 64 heads over 8 of 64, with append, 133 MB: 32 us; 4 blocks of 96 .. 288: 8 us.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <type_traits>

#include "cache_q8.cuh"
#include "cpa_tcgen05.cuh"
#include "ring.h"

namespace {

constexpr int kCons = 4;                              // consumer warps (the merger counts on four: four times eight heads are its lanes)
constexpr int kProducer = kCons, kMerger = kCons + 1;  // the other two warps
constexpr int kQ8Threads = (kCons + 2) * 32;
constexpr int kCtasPerSm = 2;
constexpr int kStages = 3;
constexpr int kAhead = 2;                             // rounds that the producer looks ahead
constexpr uint32_t kLongSpin = 1u << 24;              // waits that last for a whole range of pages
constexpr uint32_t kQ8Spin = 1u << 18;                // bounded waits (each try suspends briefly)
constexpr float kBase = 6.f, kSlack = 9.f;            // weights: 2^kBase at the maximum, up to 2^(kBase + kSlack) above it
// What the running maxima start from.  Finite, so that scores of -inf (beyond fp32, or of a V scale of zero) less a maximum
// that has met nothing else are -inf and their weights zero; a row of nothing else is 0 / 0, NaN, as a softmax's is.
constexpr float kLowest = -FLT_MAX;

template <int D>
struct Q8Shape {
    static constexpr int TP = D == 128 ? 2 : 4;       // pages per consumer warp and round
    static constexpr int kRound = kCons * TP;         // pages of a round
    // What starting and ending a (block, kv head) costs, in pages: the cut counts it, so that CTAs with many short blocks
    // get fewer pages (192 short sequences: 62.5 us without, 59.8 at 10, 57.4 at 12, 58.1 at 20; at head_dim 64, 16 blocks
    // of 8192 with 8 kv heads: 33.5 at 6, 31.9 at 12, 31.5 at 18 and 24, and 16 blocks of 96 .. 288: 12.4 at 6, 8.9 from
    // 12 to 24, 9.4 at 30).
    static constexpr int kUnitCost = D == 128 ? 12 : 18;
    static constexpr int kPageBytes = 2 * kPage * D;  // K and V codes of a (page, kv head)
    static constexpr int kData = kRound * kPageBytes;
    // behind a stage's pages: queries, the new K and V rows, scales, the round's descriptor, and (max, sum, max) of the
    // four warps for the merge
    static constexpr int kQ = 0, kNew = kQ + 8 * D * 2, kScale = kNew + 2 * D * 2, kDesc = (kScale + kRound * 8 + 15) / 16 * 16,
                         kMl = kDesc + 48, kMeta = (kMl + kCons * 8 * 16 + 127) / 128 * 128;
    static constexpr int kSmem = kStages * (kData + kMeta) + 1024;
};

struct round_desc {
    int b, g, page0, n;       // pages [page0, page0 + n) of block b, kv head g; n == 0: the end
    int flags;                // 1: first round of the segment, 2: last, 4: the last page takes the new row
    int len;                  // the block's tokens, the new one included
    int first, parts;         // the first of the CTAs that share the (block, kv head), and how many they are
};

// CTA r leaves a partial of a (block, kv head) that began before its range in slot 2 r, of one that begins in it and
// goes on in 2 r + 1.
__device__ __forceinline__ int slot_of(int r, int first) { return 2 * r + (r == first); }

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
template <int IMM>
__device__ __forceinline__ uint4 lds16_at(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4 + %5];\n" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a), "n"(IMM));
    return r;
}
template <int IMM>
__device__ __forceinline__ uint2 lds8_at(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2 + %3];\n" : "=r"(r.x), "=r"(r.y) : "r"(a), "n"(IMM));
    return r;
}
__device__ __forceinline__ void sts16(uint32_t a, int x, int y, int z, int w) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};\n" :: "r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
// body(0), body(1), ... with the number as a constant
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F&& body) {
    if constexpr (I < N) {
        body(std::integral_constant<int, I>{});
        static_for<N, I + 1>(body);
    }
}
__device__ __forceinline__ float ex2(float x) {
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(d) : "f"(x));
    return d;
}
// product rounded towards zero, which keeps subnormals and never gives an infinity of finite factors
__device__ __forceinline__ float mul_down(float a, float b) {
    float d;
    asm("mul.rz.f32 %0, %1, %2;\n" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Whether a phase has completed, without the pause of a try.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }
// four codes to two f16 pairs (the halves are named inside the assembly: taken apart in C++ each costs an instruction)
struct f16x4 { uint32_t lo, hi; };
__device__ __forceinline__ f16x4 to_f16x4(uint32_t w) {
    f16x4 r;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}\n"
        : "=r"(r.lo), "=r"(r.hi) : "r"(w));
    return r;
}

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
__device__ __forceinline__ int block_len(int b, const q8_tables& t, const int32_t* lens, const int32_t* active, int append,
                                         int& ip, int& status) {
    // (all loads first, so that those of several blocks can be in flight together)
    const int len = ld_i32(lens + b), first = ld_i32(t.page_indptr + b), end = ld_i32(t.page_indptr + b + 1),
              on = active ? ld_i32(active + b) : 1;
    ip = first;
    status = on == 0 ? 0 : len < 0 ? kStatusInvalid : (int64_t)len + append > (int64_t)(end - first) * kPage ? kStatusNoSpace : 0;
    return on == 0 || status ? -1 : len + append;
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
    int min_quota;             // cells of a range at least
    int slots;                 // partial slots of the workspace
    int list_len;              // entries of the page list, in use or not
};

// Stores a finished row pair: dims d, d + 1 of query head h.
__device__ __forceinline__ void store_pair(const q8_args& a, int b, int g, int h, int D, int d, float o0, float o1, float L,
                                           float Mo, float Ml) {
    // the factor 2^(Mo - kBase - Ml) in two halves: on its own it may leave fp32's range where the result does not; the
    // last product may be subnormal, as bf16 values go down to 2^-133
    const float e = ex2(0.5f * (Mo - kBase - Ml)), inv = 1.f / L;
    *reinterpret_cast<__nv_bfloat162*>(a.o + ((int64_t)b * a.Hq + g * a.G + h) * D + d) =
        __floats2bfloat162_rn(mul_keep(o0 * inv * e, e), mul_keep(o1 * inv * e, e));
}

__device__ __forceinline__ float4* partial_ml(const q8_args& a, int D) {
    return reinterpret_cast<float4*>(a.ws + (int64_t)a.slots * a.G * D);
}
// Where a consumer leaves dims 2u, 2u + 1 of head h inside its 8 x D floats: neither it nor the merger meets a bank twice.
template <int D>
__device__ __forceinline__ int dump_at(int h, int u) {
    const int x = D == 128 ? ((u >> 4) & 1) << 2 : 0;
    return (h * (D / 2) + (u ^ x ^ (h >> 1))) * 8;
}

// Joins the partials of a (block, kv head), for the heads of one task (128 floats: one head of 128, two of 64), by one
// warp.  Lane i of a head's D / 4 lanes holds the factors of partial i of a batch and four dimensions of the result.
template <int D>
__device__ __forceinline__ void join_partials(const q8_args& a, int blk, int head, int first, int parts, int task, int lane) {
    // partials of a batch, at most HL (20: the 37 of a head of one long block take two batches, 50.0 us for 50.5)
    constexpr int HL = D / 4, kJoin = D == 128 ? 20 : 16;
    const int sub = lane % HL, h = task * (32 / HL) + lane / HL;
    const bool there = h < a.G;
    const float4* ws_ml = partial_ml(a, D);
    float Ml = -INFINITY, Mo = -INFINITY, L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int at = 0; at < parts; at += kJoin) {
        float4 m = make_float4(-INFINITY, 0.f, -INFINITY, 0.f), x[kJoin];
#pragma unroll
        for (int i = 0; i < kJoin; ++i)              // all loads of a batch are in flight together
            x[i] = there && at + i < parts
                       ? __ldcg(reinterpret_cast<const float4*>(a.ws + ((int64_t)slot_of(first + at + i, first) * a.G + h) * D) + sub)
                       : make_float4(0.f, 0.f, 0.f, 0.f);
        if (there && sub < kJoin && at + sub < parts) m = __ldcg(ws_ml + (int64_t)slot_of(first + at + sub, first) * a.G + h);
        float ml = m.x, mo = m.z;
#pragma unroll
        for (int w = HL / 2; w > 0; w >>= 1) {
            ml = fmaxf(ml, __shfl_xor_sync(0xffffffffu, ml, w));
            mo = fmaxf(mo, __shfl_xor_sync(0xffffffffu, mo, w));
        }
        ml = fmaxf(ml, Ml);
        mo = fmaxf(mo, Mo);
        const float fl = Ml == -INFINITY ? 0.f : ex2(Ml - ml), fo = Mo == -INFINITY ? 0.f : ex2(Mo - mo);
        Ml = ml;
        Mo = mo;
        // (lanes without a partial hold a maximum of -inf and a sum of zero)
        L = L * fl + (m.x == -INFINITY ? 0.f : ex2(m.x - Ml) * m.y);
        const float f = m.z == -INFINITY ? 0.f : ex2(m.z - Mo);
        o.x *= fo; o.y *= fo; o.z *= fo; o.w *= fo;
#pragma unroll
        for (int i = 0; i < kJoin; ++i) {
            const float fi = __shfl_sync(0xffffffffu, f, i, HL);
            o.x = fmaf(fi, x[i].x, o.x); o.y = fmaf(fi, x[i].y, o.y); o.z = fmaf(fi, x[i].z, o.z); o.w = fmaf(fi, x[i].w, o.w);
        }
    }
#pragma unroll
    for (int x = HL / 2; x > 0; x >>= 1) L += __shfl_xor_sync(0xffffffffu, L, x);
    if (there) {
        store_pair(a, blk, head, h, D, 4 * sub, o.x, o.y, L, Mo, Ml);
        store_pair(a, blk, head, h, D, 4 * sub + 2, o.z, o.w, L, Mo, Ml);
    }
}

template <int D>
__global__ void __launch_bounds__(kQ8Threads, kCtasPerSm)
decode_q8_kernel(const __grid_constant__ CUtensorMap tm, const q8_args a) {
    using Sh = Q8Shape<D>;
    constexpr int TP = Sh::TP;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) uint64_t sm_full[kStages], sm_empty[kStages], sm_dump[kStages], sm_end;
    __shared__ int sm_scan[kQ8Threads / 32], sm_strip[kQ8Threads], sm_len[kQ8Threads], sm_ip[kQ8Threads], sm_dump_stage[kStages];
    __shared__ int4 sm_final;                          // a merge that is left to all warps at the end
    __shared__ int sm_down;
    __shared__ volatile int sm_dead;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t data0 = (smem_u32(raw) + 1023u) & ~1023u, meta0 = data0 + kStages * Sh::kData;
    const uint32_t full0 = smem_u32(sm_full), empty0 = smem_u32(sm_empty), dump0 = smem_u32(sm_dump), end_bar = smem_u32(&sm_end);
    if (tid == 0) {
        // full: the producer's announcement and its lanes' scales; empty: the consumers (the merger for them)
        for (int s = 0; s < kStages; ++s) { mbar_init(full0 + 8 * s, 33); mbar_init(empty0 + 8 * s, kCons); mbar_init(dump0 + 8 * s, kCons); }
        mbar_init(end_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        fence_async();
        asm volatile("prefetch.tensormap [%0];\n" :: "l"(&tm) : "memory");
        sm_dead = 0;
    }
    // What the start is going to wait for, towards L2 while the stream's earlier work ends (a line that is still to be
    // written is updated there): lengths, page offsets and, each CTA its share, the page list.
    {
        const int64_t at = ((int64_t)blockIdx.x * kQ8Threads + tid) * 32;
        if (at < a.list_len) asm volatile("prefetch.global.L2 [%0];\n" :: "l"(a.t.page_indices + at));
        if (at < a.B) {
            asm volatile("prefetch.global.L2 [%0];\n" :: "l"(a.lens + at));
            asm volatile("prefetch.global.L2 [%0];\n" :: "l"(a.t.page_indptr + at));
        }
    }
    // the next launch of the stream may be made ready now (it waits as this one does)
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    // everything above touches nothing that an earlier launch writes; this one may have been started before that one ended
    asm volatile("griddepcontrol.wait;\n" ::: "memory");

    // ---- the cut: every thread takes a strip of blocks, and the strips' page counts are scanned
    const int append = a.k_new != nullptr;
    const int run = (a.B + kQ8Threads - 1) / kQ8Threads, b_lo = min(a.B, tid * run), b_hi = min(a.B, b_lo + run);
    int mine = 0, my_len = -1, my_ip = 0, first_len = 0;
#pragma unroll 4
    for (int b = b_lo; b < b_hi; ++b) {
        int status;
        my_len = block_len(b, a.t, a.lens, a.active, append, my_ip, status);
        if (my_len > 0 && mine == 0) first_len = my_len;
        if (my_len > 0) mine += (my_len + kPage - 1) / kPage + Sh::kUnitCost;
    }
    // this CTA keeps the books of every gridDim-th block: status, new length, and the zero row of an empty block
    for (int64_t b = blockIdx.x + (int64_t)gridDim.x * tid; b < a.B; b += (int64_t)gridDim.x * kQ8Threads) {
        int ip, status;
        const int len = block_len((int)b, a.t, a.lens, a.active, append, ip, status);
        if (status) atomicCAS(a.t.header, 0, status);
        if (a.lens_out) a.lens_out[b] = len < 0 ? ld_i32(a.lens + b) : len;
        if (len == 0)
            for (int i = 0; i < a.Hq * (D / 8); ++i)
                reinterpret_cast<uint4*>(a.o + b * a.Hq * D)[i] = make_uint4(0, 0, 0, 0);
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
    sm_strip[tid] = before + inc - mine;               // pages of the blocks in front of the strip
    if (mine > 0 && before + inc == mine) sm_down = first_len & 1;   // (one thread: the first strip that holds any)
    if (tid < a.B && run == 1) { sm_len[tid] = my_len; sm_ip[tid] = my_ip; }
    const int64_t all = (int64_t)total * a.Hkv;
    const int64_t quota = max((all + gridDim.x - 1) / (int64_t)gridDim.x, (int64_t)a.min_quota);
    const int64_t x0 = quota * blockIdx.x;
    if (x0 >= all) return;                             // (uniform) more CTAs than work
    __syncthreads();

    const int tasks = (a.G * D + 127) / 128;           // of join_partials
    bool dead = false;
    // A wait that gives up ends the warp, and by the flag those that wait for it; every wait is bounded by itself too.
    auto wait = [&](uint32_t bar, uint32_t parity) {
        mbar_wait(bar, parity, dead, a.t.header, kQ8Spin);
        if (__any_sync(0xffffffffu, dead)) { dead = true; sm_dead = 1; }
        return !dead;
    };
    auto long_wait = [&](uint32_t bar, uint32_t parity) {
        uint32_t spins = 0;
        while (!dead && !mbar_try_wait(bar, parity))
            if ((++spins & 1023u) == 0 && (sm_dead || spins > kLongSpin)) { dead = true; atomicCAS(a.t.header, 0, kStatusWaitGaveUp); }
        if (__any_sync(0xffffffffu, dead)) { dead = true; sm_dead = 1; }
        return !dead;
    };

    if (warp == kProducer) {
        // ================================================================ producer
        // A window of 32 blocks in the lanes' registers: tokens and first entry of the page list.
        int win = 0, w_len, w_ip;
        auto window = [&]() {
            int status;
            w_len = -1;
            w_ip = 0;
            if (win + lane >= a.B) return;
            if (run == 1) { w_len = sm_len[win + lane]; w_ip = sm_ip[win + lane]; }
            else w_len = block_len(win + lane, a.t, a.lens, a.active, append, w_ip, status);
        };
        int b = 0, g = 0, len = 0, ip = 0, pages = 0;
        // Consecutive steps walk the pages in opposite directions (the first block's length says which), so that what a
        // step has read last, and L2 still holds, is what the next one reads first.
        const bool down = sm_down != 0;
        const int64_t x1 = min(x0 + quota, all), x = down ? x1 - 1 : x0;
        int64_t unit0 = 0;                              // where the unit starts
        int pb = 0, pe = 0;                             // its pages inside the range that are still to hand out
        bool opened = false;                            // a round of this unit has been handed out
        int parts = 0, first = 0;
        auto clip = [&]() {
            pages = (len + kPage - 1) / kPage;
            pb = (int)max((int64_t)0, x0 - unit0);
            pe = (int)min((int64_t)pages, x1 - unit0);
            opened = false;
        };
        // to the cell that the walk starts at: the strip that holds it, the block in the strip, head and page in the block
        auto locate = [&]() {
            int lo = 0, hi = kQ8Threads - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if ((int64_t)sm_strip[mid] * a.Hkv <= x) lo = mid; else hi = mid - 1;
            }
            int64_t at = (int64_t)sm_strip[lo] * a.Hkv;
            win = lo * run;
            for (;;) {
                window();
                int sum = w_len > 0 ? (w_len + kPage - 1) / kPage + Sh::kUnitCost : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, sum, o);
                    if (lane >= o) sum += v;
                }
                const uint32_t past = __ballot_sync(0xffffffffu, at + (int64_t)sum * a.Hkv > x);
                if (past) {
                    const int l = __ffs(past) - 1;
                    b = win + l;
                    len = __shfl_sync(0xffffffffu, w_len, l);
                    ip = __shfl_sync(0xffffffffu, w_ip, l);
                    const int cells = (len + kPage - 1) / kPage + Sh::kUnitCost;
                    const int64_t in = x - at - (int64_t)(__shfl_sync(0xffffffffu, sum, l) - cells) * a.Hkv;
                    g = (int)(in / cells);
                    unit0 = x - in % cells;
                    clip();
                    return;
                }
                at += (int64_t)__shfl_sync(0xffffffffu, sum, 31) * a.Hkv;
                win += 32;
                if (win >= a.B) return;                  // (cannot be reached: the walk starts inside the blocks)
            }
        };
        locate();
        // the next round into `r`, and each lane's page of it
        auto next = [&](round_desc& r, int& id) {
            r.n = 0;
            while (pb >= pe) {                          // on to the next (block, kv head) that has pages in the range
                if (down ? unit0 <= x0 : unit0 + pages + Sh::kUnitCost >= x1) return;
                const int from = pages;
                g += down ? -1 : 1;
                if (g < 0 || g == a.Hkv) {
                    g = down ? a.Hkv - 1 : 0;
                    do {
                        b += down ? -1 : 1;
                        if (b < 0 || b >= a.B) { pb = pe = 0; unit0 = down ? x0 : x1; return; }   // (cannot be reached)
                        if (b < win || b >= win + 32) { win = down ? max(b - 31, 0) : b; window(); }
                        len = __shfl_sync(0xffffffffu, w_len, b - win);
                    } while (len <= 0);
                    ip = __shfl_sync(0xffffffffu, w_ip, b - win);
                }
                unit0 += down ? -((len + kPage - 1) / kPage + Sh::kUnitCost) : from + Sh::kUnitCost;
                clip();
            }
            r.flags = 0;
            if (!opened) {
                first = (int)(unit0 / quota);
                parts = (int)((unit0 + pages - 1) / quota) - first + 1;
                r.flags = 1;
                opened = true;
            }
            r.b = b;
            r.g = g;
            r.n = min(pe - pb, Sh::kRound);
            r.page0 = down ? pe - r.n : pb;
            r.len = len;
            r.first = first;
            r.parts = parts;
            id = lane < r.n ? ld_i32(a.t.page_indices + ip + r.page0 + lane) : 0;
            (down ? pe : pb) += down ? -r.n : r.n;
            r.flags |= (pb >= pe ? 2 : 0) | (append && r.page0 + r.n == pages ? 4 : 0);
        };
        // Descriptors and page ids run kAhead rounds in front of the copies, so that no load is waited for.
        round_desc d[kAhead + 1];
        int id[kAhead + 1];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next(d[i], id[i]);
        int it = 0;
        for (;; ++it) {
            next(d[kAhead], id[kAhead]);
            const int st = it % kStages;
            if (it >= kStages && !wait(empty0 + 8 * st, (uint32_t)(it / kStages - 1) & 1u)) break;
            const uint32_t data = data0 + st * Sh::kData, meta = meta0 + st * Sh::kMeta, bar = full0 + 8 * st;
            const int cell = id[0] * a.Hkv + d[0].g;    // (page, kv head)
            const int last_cell = __shfl_sync(0xffffffffu, cell, d[0].n > 0 ? d[0].n - 1 : 0);
            if (lane == 0) {
                sts16(meta + Sh::kDesc, d[0].b, d[0].g, d[0].page0, d[0].n);
                sts16(meta + Sh::kDesc + 16, d[0].flags, d[0].len, d[0].first, d[0].parts);
                sts16(meta + Sh::kDesc + 32, last_cell, 0, 0, 0);
                if (d[0].n > 0)
                    mbar_expect_tx(bar, d[0].n * Sh::kPageBytes + (d[0].flags & 1 ? a.G * D * 2 : 0) + (d[0].flags & 4 ? 2 * D * 2 : 0));
                else
                    mbar_arrive(bar);                   // the end: no copies
            }
            __syncwarp();
            if (lane < d[0].n) {
                tma_load_2d(data + lane * Sh::kPageBytes, &tm, 0, cell * (Sh::kPageBytes / 128), bar);
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n"
                             :: "r"(meta + Sh::kScale + 8 * lane), "l"(a.scales + (int64_t)cell * 2) : "memory");
            }
            // every lane's arrival, once its scale has landed
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];\n" :: "r"(bar) : "memory");
            if (d[0].n == 0) break;
            if (lane == 0) {
                if (d[0].flags & 1) bulk_copy(meta + Sh::kQ, a.q + ((int64_t)d[0].b * a.Hq + d[0].g * a.G) * D, a.G * D * 2, bar);
                if (d[0].flags & 4) {
                    const int64_t row = ((int64_t)d[0].b * a.Hkv + d[0].g) * D;
                    bulk_copy(meta + Sh::kNew, a.k_new + row, D * 2, bar);
                    bulk_copy(meta + Sh::kNew + D * 2, a.v_new + row, D * 2, bar);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) { d[i] = d[i + 1]; id[i] = id[i + 1]; }
        }
        // See the copies in flight through before leaving: the consumers do so by using them, but not when one of their
        // waits has given up, which this warp need not have met.
        if (lane == 0) {
            const ring_rounds left = ring_in_flight(it, kStages, !dead);
            for (int i = left.first; i < left.end; ++i)
                mbar_drain(full0 + 8 * (i % kStages), (uint32_t)(i / kStages) & 1u, kDrainLimit);
        }
        __syncwarp();
        return;
    }

    if (warp == kMerger) {
        // ================================================================ merger
        for (int k = 0;; ++k) {
            if (!long_wait(dump0 + 8 * (k % kStages), (uint32_t)(k / kStages) & 1u)) return;
            const int st = sm_dump_stage[k % kStages];
            if (st < 0) break;
            const uint32_t data = data0 + st * Sh::kData, meta = meta0 + st * Sh::kMeta;
            const uint4 e0 = lds16(meta + Sh::kDesc), e1 = lds16(meta + Sh::kDesc + 16);
            const int blk = (int)e0.x, head = (int)e0.y, first = (int)e1.z, parts = (int)e1.w;
            const int64_t row0 = (int64_t)slot_of((int)blockIdx.x, first) * a.G;
            // lane (w, h): consumer w's factor of head h, and with the other lanes of h the head's maxima and sum
            const uint4 x = lds16(meta + Sh::kMl + lane * 16);
            const float ml = __uint_as_float(x.x), l = __uint_as_float(x.y), mo = __uint_as_float(x.z);
            float Ml = fmaxf(ml, __shfl_xor_sync(0xffffffffu, ml, 8)), Mo = fmaxf(mo, __shfl_xor_sync(0xffffffffu, mo, 8));
            Ml = fmaxf(Ml, __shfl_xor_sync(0xffffffffu, Ml, 16));
            Mo = fmaxf(Mo, __shfl_xor_sync(0xffffffffu, Mo, 16));
            // (a consumer that had no page holds zeros under the lowest maximum)
            float f = ex2(mo - Mo), L = ex2(ml - Ml) * l;
            L += __shfl_xor_sync(0xffffffffu, L, 8);
            L += __shfl_xor_sync(0xffffffffu, L, 16);
            // The finished row's factor 2^(Mo - kBase - Ml) / L goes in two halves: on its own it may leave fp32's range
            // where the result does not (the last product keeps subnormals, as in store_pair).
            const float e = parts == 1 ? ex2(0.5f * (Mo - kBase - Ml)) : 1.f;
            if (parts == 1) f *= 1.f / L;
            else if (lane < a.G) partial_ml(a, D)[row0 + lane] = make_float4(Ml, L, Mo, 0.f);
#pragma unroll 4
            for (int h = 0; h < a.G; ++h) {
                float fw[kCons];
#pragma unroll
                for (int w = 0; w < kCons; ++w) fw[w] = __shfl_sync(0xffffffffu, f, 8 * w + h);
                const float eh = __shfl_sync(0xffffffffu, e, h);
#pragma unroll
                for (int i = 0; i < D / 64; ++i) {
                    const int u = lane + 32 * i;
                    float o0 = 0.f, o1 = 0.f;
#pragma unroll
                    for (int w = 0; w < kCons; ++w) {
                        const uint2 y = lds8(data + w * Sh::kPageBytes + dump_at<D>(h, u));
                        o0 = fmaf(fw[w], __uint_as_float(y.x), o0);
                        o1 = fmaf(fw[w], __uint_as_float(y.y), o1);
                    }
                    if (parts == 1)
                        *reinterpret_cast<__nv_bfloat162*>(a.o + ((int64_t)blk * a.Hq + head * a.G + h) * D + 2 * u) =
                            __floats2bfloat162_rn(mul_keep(o0 * eh, eh), mul_keep(o1 * eh, eh));
                    else
                        *reinterpret_cast<float2*>(a.ws + (row0 + h) * D + 2 * u) = make_float2(o0, o1);
                }
            }
            __syncwarp();
            if (lane < kCons) mbar_arrive(empty0 + 8 * st);      // for the four consumers
            if (parts == 1) continue;
            // One atomic publishes this partial (the lanes' stores come before it by the warp barrier) and, for the one who
            // finds all others counted, makes theirs visible.  The counter is back at zero after the last.
            unsigned before_me = 0;
            __syncwarp();
            if (lane == 0)
                asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;\n" : "=r"(before_me)
                             : "l"(a.t.tickets + (int64_t)blk * a.Hkv + head), "r"(parts - 1) : "memory");
            before_me = __shfl_sync(0xffffffffu, before_me, 0);
            if (before_me != (unsigned)parts - 1) continue;
            __syncwarp();
            // The last one in joins the partials: at the end of the CTA's work with all warps, else in the background.
            const int nk = k + 1;
            bool end = false;
            if (mbar_test(dump0 + 8 * (nk % kStages), (uint32_t)(nk / kStages) & 1u)) end = sm_dump_stage[nk % kStages] < 0;
            end = __all_sync(0xffffffffu, end);
            if (end) {
                if (lane == 0) { sm_final = make_int4(blk, head, first, parts); mbar_arrive(end_bar); }
                for (int task = kCons; task < tasks; task += kCons + 1) join_partials<D>(a, blk, head, first, parts, task, lane);
                return;
            }
            for (int task = 0; task < tasks; ++task)
                join_partials<D>(a, blk, head, first, parts, task, lane);
        }
        if (lane == 0) { sm_final = make_int4(0, 0, 0, 0); mbar_arrive(end_bar); }
        return;
    }

    // ==================================================================== consumers
    const int g8 = lane >> 2, t4 = lane & 3;
    int segment = 0;
    // this lane's places in a page (its own first page of a round): K rows key(g) and key(g + 8), V rows key(2t) ...
    const uint32_t own_page = warp * Sh::kPageBytes;
    uint32_t k_off[2], v_off[4];
    if (D == 128) {                                     // rows 8 apart have the same swizzle, the other piece has not
        k_off[0] = own_page + piece_at<D>(key_of_row<D>(g8), t4);
        k_off[1] = own_page + piece_at<D>(key_of_row<D>(g8), t4 + 4);
    } else {
        k_off[0] = own_page + piece_at<D>(key_of_row<D>(g8), t4);
        k_off[1] = own_page + piece_at<D>(key_of_row<D>(g8 + 8), t4);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int key = key_of_row<D>(2 * t4 + (r & 1) + 8 * (r >> 1));
        v_off[r] = own_page + (D == 128 ? piece_at<D>(key, g8) : piece_at<D>(key, g8 >> 1) + (g8 & 1) * 8);
    }
    uint32_t qf[D / 64][4][2];
    float acc[D / 16][4], c0 = 0.f, c1 = 0.f;           // c: what a score's sum is multiplied with, for heads 2t, 2t + 1
    float ml0 = kLowest, ml1 = kLowest, mo0 = kLowest, mo1 = kLowest, l0 = 0.f, l1 = 0.f;

    for (int it = 0;; ++it) {
        const int st = it % kStages;
        const uint32_t data = data0 + st * Sh::kData, meta = meta0 + st * Sh::kMeta;
        if (!wait(full0 + 8 * st, (uint32_t)(it / kStages) & 1u)) return;
        const uint4 e0 = lds16(meta + Sh::kDesc), e1 = lds16(meta + Sh::kDesc + 16);
        const int page0 = (int)e0.z, n = (int)e0.w, flags = (int)e1.x, len = (int)e1.y;
        if (n == 0) break;
        if (flags & 1) {
            // the queries as f16 B fragments: contracted elements 2t, 2t+1, 2t+8, 2t+9 of step (p, w) are dimensions
            // 64 p + 16 t + 4 w + 0 .. 3.  2^7 at the row's largest element.
            uint4 v[D / 64][2];
            uint32_t two = 0;                                // largest magnitudes, as bf16 bits in two halves
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    v[p][i] = g8 < a.G ? lds16(meta + Sh::kQ + (g8 * D + 64 * p + 16 * t4 + 8 * i) * 2) : make_uint4(0, 0, 0, 0);
                    two = __vmaxu2(__vmaxu2(two, __vmaxu2(v[p][i].x & 0x7FFF7FFFu, v[p][i].y & 0x7FFF7FFFu)),
                                   __vmaxu2(v[p][i].z & 0x7FFF7FFFu, v[p][i].w & 0x7FFF7FFFu));
                }
            two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, 1));
            two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, 2));
            const int amax = (int)max(two & 0xFFFFu, two >> 16);
            int e = amax >> 7;                               // biased exponent; infinities and NaN go through as they are
            e = amax == 0 || e == 255 ? 134 : max(e, 8);
            const float down = __uint_as_float((uint32_t)(e - 7) << 23);
            const uint32_t up2 = (uint32_t)(261 - e) << 7 | (uint32_t)(261 - e) << 23;     // a bf16 pair
#pragma unroll
            for (int p = 0; p < D / 64; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t w[4] = {v[p][i].x, v[p][i].y, v[p][i].z, v[p][i].w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t x;                          // (exact, and what becomes subnormal is below f16's range)
                        asm("mul.rn.bf16x2 %0, %1, %2;\n" : "=r"(x) : "r"(w[j]), "r"(up2));
                        qf[p][2 * i + (j >> 1)][j & 1] = pack_f16(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
                    }
                }
            const float c = mul_keep(down, a.scale_log2);
            c0 = __shfl_sync(0xffffffffu, c, 8 * t4);
            c1 = __shfl_sync(0xffffffffu, c, 8 * t4 + 4);
            ml0 = ml1 = mo0 = mo1 = kLowest;
            l0 = l1 = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
        }
        const int n_mine = (n - warp + kCons - 1) / kCons;   // this warp's pages of the round (may be 0)
        bool wrote = false;                                  // into the stage: the copy that refills it has to come after

        if ((flags & 4) && n_mine > 0 && warp + kCons * (n_mine - 1) == n - 1) {
            // ---- the block's newest page is this warp's: quantise the new row into it, here and in the pool
            const int slot = (len - 1) % kPage, j = n - 1;
            const uint32_t chunk0 = data + j * Sh::kPageBytes;
            const int64_t cell = (int64_t)(int)lds16(meta + Sh::kDesc + 32).x;       // page * Hkv + g
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
                        const float f = mul_keep(old, q8_inverse(s));   // (another writer's scale may be subnormal)
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
                const bool p2 = q8_power_of_two(s);
                uint32_t codes = to_e4m3x2(q8_divide(x[0], s, p2), q8_divide(x[1], s, p2));
                if (D == 128) codes |= to_e4m3x2(q8_divide(x[D / 32 - 2], s, p2), q8_divide(x[D / 32 - 1], s, p2)) << 16;
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
            wrote = true;
            __syncwarp();
        }

        // ---- slots behind the block's tokens may hold anything, a NaN among it that a weight of zero would not silence
        const int cut_page = warp + kCons * (n_mine - 1), cut_at = len - (page0 + cut_page) * kPage;
        if (n_mine > 0 && cut_at < kPage) {
            for (int i = lane; i < (kPage - cut_at) * (D / 16); i += 32) {
                const int r = cut_at + i / (D / 16);
                sts16(data + cut_page * Sh::kPageBytes + kPage * D + piece_at<D>(r, i % (D / 16)), 0, 0, 0, 0);
            }
            wrote = true;
            __syncwarp();
        }
        // ---- scores of this warp's pages: s[i] = (key(g), head 2t), (key(g), 2t+1), (key(g+8), 2t), (key(g+8), 2t+1)
        float s[TP][4], lv[TP];
        float hi0 = -INFINITY, hi1 = -INFINITY, ho0 = -INFINITY, ho1 = -INFINITY;
        const uint32_t ka = data + k_off[0], kb = data + k_off[1];
        static_for<TP>([&](auto ic) {
            constexpr int i = decltype(ic)::value, at = kCons * i * Sh::kPageBytes;
            if (i >= n_mine) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][e] = -INFINITY;
                lv[i] = 0.f;
                return;
            }
            const int j = warp + kCons * i;
            const uint2 sc = lds8(meta + Sh::kScale + 8 * j);
            // rows key(g) and key(g + 8); at 128, pieces t and t + 4 of each
            const uint4 r0 = lds16_at<at>(ka), r1 = D == 128 ? lds16_at<at + 1024>(ka) : lds16_at<at>(kb);
            const uint4 r2 = D == 128 ? lds16_at<at>(kb) : r0, r3 = D == 128 ? lds16_at<at + 1024>(kb) : r1;
            const uint32_t w0[8] = {r0.x, r0.y, r0.z, r0.w, r2.x, r2.y, r2.z, r2.w};
            const uint32_t w1[8] = {r1.x, r1.y, r1.z, r1.w, r3.x, r3.y, r3.z, r3.w};
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < D / 16; ++w) {
                const f16x4 x0 = to_f16x4(w0[w]), x1 = to_f16x4(w1[w]);
                mma_f16(sum, x0.lo, x1.lo, x0.hi, x1.hi, qf[w >> 2][w & 3][0], qf[w >> 2][w & 3][1]);
            }
            // (either factor may be subnormal; rounded towards zero a product that passes fp32's range stays finite, so that
            // keys of zeros score zero there too)
            const float ks = __uint_as_float(sc.x), k0 = mul_down(ks, c0), k1 = mul_down(ks, c1);
            s[i][0] = sum[0] * k0;
            s[i][1] = sum[1] * k1;
            s[i][2] = sum[2] * k0;
            s[i][3] = sum[3] * k1;
            // (zero gives -inf: the page takes part in the sums with weights of zero; scales below the normal range count)
            asm("lg2.approx.f32 %0, %1;\n" : "=f"(lv[i]) : "f"(__uint_as_float(sc.y)));
            if (j == cut_page && cut_at < kPage) {
                if (key_of_row<D>(g8) >= cut_at) s[i][0] = s[i][1] = -INFINITY;
                if (key_of_row<D>(g8 + 8) >= cut_at) s[i][2] = s[i][3] = -INFINITY;
            }
            const float a0 = fmaxf(s[i][0], s[i][2]), a1 = fmaxf(s[i][1], s[i][3]);
            hi0 = fmaxf(hi0, a0);
            hi1 = fmaxf(hi1, a1);
            ho0 = fmaxf(ho0, a0 + lv[i]);
            ho1 = fmaxf(ho1, a1 + lv[i]);
        });
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
                    const float up = fmaxf(m, hi), f = ex2(m - up);
                    m = up;
                    return f;
                };
                l0 *= raise(ml0, hi0);
                l1 *= raise(ml1, hi1);
                const float f0 = raise(mo0, ho0), f1 = raise(mo1, ho1);
                if (!(flags & 1))                            // (a segment's first round finds zeros)
#pragma unroll
                for (int j = 0; j < D / 16; ++j) { acc[j][0] *= f0; acc[j][1] *= f1; acc[j][2] *= f0; acc[j][3] *= f1; }
            }
            // ---- weights, and O^T += V^T P^T
            const float b0 = kBase - mo0, b1 = kBase - mo1;
            uint32_t va[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) va[r] = data + v_off[r];
            static_for<TP>([&](auto ic) {
                constexpr int i = decltype(ic)::value, at = kCons * i * Sh::kPageBytes + kPage * D;
                if (i >= n_mine) return;
                l0 += ex2(s[i][0] - ml0) + ex2(s[i][2] - ml0);
                l1 += ex2(s[i][1] - ml1) + ex2(s[i][3] - ml1);
                const float u0 = b0 + lv[i], u1 = b1 + lv[i];
                const uint32_t p0 = transpose8(pack_f16(ex2(s[i][0] + u0), ex2(s[i][1] + u1)));
                const uint32_t p1 = transpose8(pack_f16(ex2(s[i][2] + u0), ex2(s[i][3] + u1)));
                constexpr int W = D / 32;                    // words of codes per lane and key
                uint32_t v[4][W];                            // keys key(2t), key(2t + 1), key(2t + 8), key(2t + 9)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if constexpr (D == 128) {
                        const uint4 x = r < 2 ? lds16_at<at>(va[r]) : lds16_at<at + 1024>(va[r - 2]);
                        v[r][0] = x.x; v[r][1] = x.y; v[r][2] = x.z; v[r][3] = x.w;
                    } else {
                        const uint2 x = lds8_at<at>(va[r]);
                        v[r][0] = x.x; v[r][1] = x.y;
                    }
                }
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    // codes of two keys side by side: (dims 0, 1 of the word) and (dims 2, 3)
                    const uint32_t a01 = __byte_perm(v[0][w], v[1][w], 0x5140), a23 = __byte_perm(v[0][w], v[1][w], 0x7362);
                    const uint32_t b01 = __byte_perm(v[2][w], v[3][w], 0x5140), b23 = __byte_perm(v[2][w], v[3][w], 0x7362);
                    const f16x4 xa = to_f16x4(a01), xb = to_f16x4(b01), ya = to_f16x4(a23), yb = to_f16x4(b23);
                    mma_f16(acc[2 * w], xa.lo, xa.hi, xb.lo, xb.hi, p0, p1);
                    mma_f16(acc[2 * w + 1], ya.lo, ya.hi, yb.lo, yb.hi, p0, p1);
                }
            });
        }
        if (!(flags & 2)) {
            if (wrote) fence_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(empty0 + 8 * st);
            continue;
        }

        __syncwarp();                                        // every lane has read its pages
        // ---- the segment is done: leave O and the sums to the merger, over this warp's first page of the round
        l0 += __shfl_xor_sync(0xffffffffu, l0, 4);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 4);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 8);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 8);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 16);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 16);
        const uint32_t mine_o = data + warp * Sh::kPageBytes;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const int u = g8 * (D / 16) + j;                 // dims 2u, 2u + 1 = rows g, g + 8 of tile j
            asm volatile("st.shared.v2.f32 [%0], {%1,%2};\n" :: "r"(mine_o + dump_at<D>(2 * t4, u)), "f"(acc[j][0]), "f"(acc[j][2]) : "memory");
            asm volatile("st.shared.v2.f32 [%0], {%1,%2};\n" :: "r"(mine_o + dump_at<D>(2 * t4 + 1, u)), "f"(acc[j][1]), "f"(acc[j][3]) : "memory");
        }
        if (g8 == 0) {
            const uint32_t to = meta + Sh::kMl + (warp * 8 + 2 * t4) * 16;
            asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%3};\n" :: "r"(to), "f"(ml0), "f"(l0), "f"(mo0) : "memory");
            asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%3};\n" :: "r"(to + 16), "f"(ml1), "f"(l1), "f"(mo1) : "memory");
        }
        // Entry `segment` of the merger's queue.  Its place is free: the entry before it in that place belonged to a
        // segment whose stage has been handed back, or this one could not have got one.
        if (warp == 0 && lane == 0) sm_dump_stage[segment % kStages] = st;
        fence_async();                                       // the copy that refills the stage comes after these stores
        __syncwarp();
        if (lane == 0) mbar_arrive(dump0 + 8 * (segment % kStages));
        ++segment;
    }
    // ---- the end: tell the merger, and help it with what it finds to be joined last
    if (warp == 0 && lane == 0) sm_dump_stage[segment % kStages] = -1;
    __syncwarp();
    if (lane == 0) mbar_arrive(dump0 + 8 * (segment % kStages));
    if (!long_wait(end_bar, 0)) return;
    const int4 fin = sm_final;
    if (fin.w > 0)
        for (int task = warp; task < tasks; task += kCons + 1)
            join_partials<D>(a, fin.x, fin.y, fin.z, fin.w, task, lane);
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

// Two partial slots per CTA.
int partial_slots(const cpa_config* cfg) {
    return 2 * kCtasPerSm * (cfg->num_sms ? cfg->num_sms : kSmsByDefault);
}

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
    // Cells of a range at least.  Short blocks want many ranges, though a round would hold them whole: 4 blocks of 96 .. 288
    // tokens, one kv head of 64, take 7.8 us at 8 and at 16, 9.3 at 24, 9.6 at 40; 16 such blocks, 8 kv heads of 128, 9.4,
    // 12.5, 11.8 and 12.5.  (One block of one such head alone would have 24: 6.1 us for 7.3.)
    a.min_quota = 8;
    a.slots = partial_slots(cfg);
    a.list_len = dims->page_capacity;
    // one wave; no more CTAs than the table's pages and blocks could keep busy
    const int64_t most = (((int64_t)dims->page_capacity + (int64_t)Sh::kUnitCost * dims->num_blocks) * cfg->num_kv_heads +
                          a.min_quota - 1) / a.min_quota;
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
    return (int64_t)partial_slots(cfg) * (cfg->num_q_heads / cfg->num_kv_heads) * (cfg->head_dim + 4) * 4;
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
