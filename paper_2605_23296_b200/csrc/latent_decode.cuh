// What the decode kernels of the latent cache share: their arguments, the even cut of all blocks' tiles into shares, and the
// ring through which a CTA's warps learn their segments.
#pragma once

#include <algorithm>
#include <atomic>

#include "latent.cuh"
#include "cpa_tcgen05.cuh"

namespace {

constexpr int kTile = 64;                       // tokens per tile
constexpr int kTilePages = kTile / kPage;
constexpr int kDecodeThreads = 512;
constexpr int kSms = 148;                       // of a B200; CTAs do not wait for one another, so any device will do
constexpr int kSegRing = 4;
constexpr int kBlockCost = 2;                   // what a block costs beside its tiles, in tiles (its queries, its output)
constexpr int kMinRange = 2;                    // cost of a CTA's share, at least: a tile and its block's own (4 blocks of 96..288 tokens: 11.3 us; 14.4 with 4)
constexpr float kLowest = -3e38f, kFirstMargin = 6.f;
constexpr uint32_t kPBytes = kTile * 128;
constexpr int kMaxSmem = 232448;                // 227 KB, what a CTA can have on sm_100

struct decode_args {
    q8_tables t;
    cpa_latent_io io;
    const uint64_t* turns;            // step: the query's positional part is turned; nullptr: taken as it is
    const int32_t *first, *lens, *active;
    // step (x given): the new token's row is made and stored first
    const __nv_bfloat16 *x, *weight;
    int64_t x_row;
    int32_t* lens_out;
    __nv_bfloat16* pool;
    float2* part_ml;                  // [slots, head groups, 64]
    float* part_o;                    // [slots, head groups, 64, L]
    int2* cuts;                       // [groups] (block, parts) of the block that starts in a group and goes on behind it
    int B, H, L, groups, head_groups, group_heads, interleaved;
    int list_words;                   // of the page list, for a look ahead
    float scale_log2, amplitude, eps;
};

// A block's part in a launch.
struct block_state { int len, ip, status; bool on; };
__device__ __forceinline__ block_state block_of(int b, const decode_args& a) {
    block_state r;
    const int before = ld_i32(a.lens + b), np0 = ld_i32(a.t.page_indptr + b), np1 = ld_i32(a.t.page_indptr + b + 1);
    const bool active = a.active == nullptr || ld_i32(a.active + b) != 0;
    const int64_t len = (int64_t)before + (a.x ? 1 : 0), room = (int64_t)(np1 - np0) * kPage;
    r.ip = np0;
    r.status = !active ? 0 : before < 0 ? kStatusInvalid : len > room ? kStatusNoSpace : 0;
    r.on = active && r.status == 0;
    r.len = r.on ? (int)len : 0;
    return r;
}

struct segment {
    int block, tile0, tiles, len;     // block -1: no more; tiles [tile0, tile0 + tiles) of a block of `len` tokens
    int ip, slot;                     // its first page in the list; partial slot, -1: the whole block
    int pad[2];
};

__device__ __forceinline__ row_recipe new_row_of(const decode_args& a) {
    return {a.weight, a.turns, a.eps, a.amplitude, a.interleaved};
}
template <int L>
__device__ __forceinline__ __nv_bfloat16* slot_of(const decode_args& a, const segment& g) {
    const int at = g.len - 1, page = ld_i32(a.t.page_indices + g.ip + at / kPage);
    return a.pool + ((int64_t)page * kPage + at % kPage) * (L + kRopeDim);
}

__device__ __forceinline__ int tiles_of(int len) { return (int)(((int64_t)len + kTile - 1) / kTile); }

// What every CTA reads first is brought to L2 ahead of the wait for the launches before (L2 is coherent: what is written until
// then is seen), the lists shared out.
__device__ __forceinline__ void look_ahead(const decode_args& a) {
    for (int64_t i = (int64_t)(threadIdx.x * gridDim.x + blockIdx.x) * 32; i < a.list_words; i += (int64_t)kDecodeThreads * gridDim.x * 32) {
        asm volatile("prefetch.global.L2 [%0];\n" :: "l"(a.t.page_indices + i));
        if (i < a.B) {
            asm volatile("prefetch.global.L2 [%0];\n" :: "l"(a.lens + i));
            asm volatile("prefetch.global.L2 [%0];\n" :: "l"(a.t.page_indptr + i));
        }
    }
}

// ---------------------------------------------------------------- the cut
// The tiles of all blocks in a row, each block's own cost in front of its tiles, are dealt to the groups in equal parts.  (A page
// list has fewer than 2^31 entries, so all costs together are below 2^29 + 3 * 2^20.)
// `total` in `used` shares of q or, the first rem ones, q + 1.
struct shares {
    int total, used, q, rem;
    __device__ __forceinline__ int start(int g) const { return q * g + min(g, rem); }
    __device__ __forceinline__ int group_of(int cost) const {
        const int big = rem * (q + 1);
        return cost < big ? cost / (q + 1) : rem + (cost - big) / q;
    }
};
struct CutShared { int cost[kDecodeThreads / 32]; };      // of each warp's run of blocks
__device__ __forceinline__ int blocks_per_thread(const decode_args& a) { return (a.B + kDecodeThreads - 1) / kDecodeThreads; }
// By all threads of a CTA, with a barrier; a thread takes its blocks one behind the other, which shows from some thousand blocks on (16 heads,
// blocks of 64 tokens: 192 blocks 12 us, 2000 46, 20000 425).  (What follows from the costs is left to the warp that hands the segments out: all of
// this runs once in a launch, and takes as long as its instructions take to arrive.)
__device__ __forceinline__ void sum_costs(const decode_args& a, CutShared& sm) {
    const int per = blocks_per_thread(a), b0 = min((int)threadIdx.x * per, a.B), b1 = min(b0 + per, a.B);
    int cost = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
        const block_state s = block_of(b, a);
        if (s.len > 0) cost += tiles_of(s.len) + kBlockCost;
    }
    cost = __reduce_add_sync(0xffffffffu, cost);
    if ((threadIdx.x & 31) == 0) sm.cost[threadIdx.x >> 5] = cost;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
}
__device__ __forceinline__ int inclusive_sum(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

// ---------------------------------------------------------------- segments
struct SegmentRing {
    segment seg[kSegRing];
    uint64_t full[kSegRing], empty[kSegRing];
};
__device__ __forceinline__ void init_ring(SegmentRing& ring, uint32_t readers) {
    for (int i = 0; i < kSegRing; ++i) {
        mbar_init(smem_u32(&ring.full[i]), 1);
        mbar_init(smem_u32(&ring.empty[i]), readers);
    }
}
// Segment i of this CTA, by a whole warp (each reader warp takes every one).
__device__ __forceinline__ segment take_segment(SegmentRing& ring, int i, bool& dead, int32_t* status) {
    mbar_wait(smem_u32(&ring.full[i % kSegRing]), (uint32_t)(i / kSegRing) & 1u, dead, status, kSpinLimit);
    dead = __any_sync(0xffffffffu, dead);
    segment s = ring.seg[i % kSegRing];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&ring.empty[i % kSegRing]));
    if (dead) s.block = -1;
    return s;
}
// The segments of group `group` in order, behind them one of block -1, by a whole warp; and the record of a block that goes on
// behind the group's share.
__device__ __forceinline__ void hand_out(const decode_args& a, const CutShared& sm, SegmentRing& ring, int group, bool record, bool& dead,
                                         int32_t* status) {
    const int lane = threadIdx.x & 31;
    int n = 0;
    int2 cut = make_int2(-1, 0);
    auto put = [&](const segment& s) {
        mbar_wait(smem_u32(&ring.empty[n % kSegRing]), ((uint32_t)(n / kSegRing) & 1u) ^ 1u, dead, status, kSpinLimit);
        ring.seg[n % kSegRing] = s;
        mbar_arrive(smem_u32(&ring.full[n % kSegRing]));
        ++n;
    };
    const int sums = inclusive_sum(lane < kDecodeThreads / 32 ? sm.cost[lane] : 0, lane);
    shares sh;
    sh.total = __shfl_sync(0xffffffffu, sums, 31);
    sh.used = max(1, min(a.groups, sh.total / kMinRange));
    sh.q = sh.total / sh.used;
    sh.rem = sh.total - sh.q * sh.used;
    if (group < sh.used && sh.total > 0) {
        const int lo = sh.start(group), hi = sh.start(group + 1);
        const int run = __popc(__ballot_sync(0xffffffffu, sums <= lo));         // the run of blocks in which the share starts
        int c = run ? __shfl_sync(0xffffffffu, sums, run - 1) : 0;
        for (int b = run * 32 * blocks_per_thread(a); b < a.B && c < hi; b += 32) {
            block_state s{0, 0, 0, false};
            if (b + lane < a.B) s = block_of(b + lane, a);
            const int tiles = tiles_of(s.len), mine = s.len > 0 ? tiles + kBlockCost : 0;
            const int at = inclusive_sum(mine, lane);
            const int first = c + at - mine + kBlockCost;          // cost at which the block's first tile lies
            c += __shfl_sync(0xffffffffu, at, 31);
            const int j0 = min(tiles, max(0, lo - first)), j1 = min(tiles, max(0, hi - first));
            uint32_t todo = __ballot_sync(0xffffffffu, s.len > 0 && j1 > j0);
            while (todo) {
                const int who = __ffs(todo) - 1;
                todo &= todo - 1;
                if (lane == who) {
                    const bool whole = j0 == 0 && j1 == tiles;
                    put({b + lane, j0, j1 - j0, s.len, s.ip, whole ? -1 : 2 * group + (j0 == 0 ? 1 : 0), {0, 0}});
                    if (j0 == 0 && j1 < tiles) cut = make_int2(b + lane, sh.group_of(first + tiles - 1) - group + 1);
                }
                n = __shfl_sync(0xffffffffu, n, who);
            }
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
    }
    if (lane == 0) put({-1, 0, 0, 0, 0, 0, {0, 0}});
    const uint32_t has = __ballot_sync(0xffffffffu, cut.x >= 0);
    const int who = has ? __ffs(has) - 1 : 0;
    if (record && lane == who) a.cuts[group] = cut;
}
// The blocks' books (status, new lengths), shared out to the CTAs, and rows of zeros for blocks without a token, by the 128 threads
// `tid` of a CTA.
__device__ __forceinline__ void keep_books(const decode_args& a, int tid) {
    const int pieces = a.L / 8;
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
        const block_state s = block_of(b, a);
        if (tid == 0) {
            if (s.status) atomicCAS(a.t.header, 0, s.status);
            if (a.x) a.lens_out[b] = s.on ? s.len : ld_i32(a.lens + b);
        }
        if (!s.on || s.len > 0) continue;
        __nv_bfloat16* o = (__nv_bfloat16*)a.io.o + b * a.io.o_block_stride;
        for (int e = tid; e < a.H * pieces; e += 128)
            *reinterpret_cast<uint4*>(o + (e / pieces) * a.io.o_head_stride + 8 * (e % pieces)) = make_uint4(0, 0, 0, 0);
    }
}

// ---------------------------------------------------------------- PTX
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];\n" :: "l"(map) : "memory"); }
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap* map, int group, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %3}], [%4];\n"
        :: "r"(dst), "l"(map), "r"(0), "r"(group), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_q(uint32_t dst, const CUtensorMap* map, int head, int block, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %2, %4}], [%5];\n"
        :: "r"(dst), "l"(map), "r"(0), "r"(head), "r"(block), "r"(bar) : "memory");
}
// Whether `x` holds in any of the 128 threads that meet at barrier `id`.
__device__ __forceinline__ bool any_of_128(int id, bool x) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
                 : "=r"(r) : "r"((uint32_t)x), "r"(id) : "memory");
    return r != 0;
}
__device__ __forceinline__ void sync_128(int id) { asm volatile("barrier.cta.sync %0, 128;\n" :: "r"(id) : "memory"); }
// 16 columns of this thread's lane
__device__ __forceinline__ void tc_ld16(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// ---------------------------------------------------------------- queries
constexpr int kLoaderBarrier = 3;       // of the 128 threads that bring the queries
// The turned positional parts of N query heads from h0 on (zeros behind the last of `heads`), to q_at(head, 16-byte piece), by
// 128 threads once turn[pair] holds the angles: a thread takes pieces r and r ^ 4 of a head, each other's partners in the half
// layout.
template <int N, class Q>
__device__ __forceinline__ void turn_queries(const decode_args& a, int block, int h0, int heads, int tid, const float2* turn, Q&& q_at) {
    const __nv_bfloat16* qr = (const __nv_bfloat16*)a.io.q_rope + block * a.io.q_rope_block_stride + h0 * a.io.q_rope_head_stride;
    constexpr int kRounds = (N * 4 + 127) / 128;
    const int r = tid & 3;
    uint4 x[kRounds], y[kRounds];
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int h = (tid >> 2) + 32 * k;
        x[k] = y[k] = make_uint4(0, 0, 0, 0);
        if (h < heads) {
            x[k] = ld_v4(qr + h * a.io.q_rope_head_stride + 8 * r);
            y[k] = ld_v4(qr + h * a.io.q_rope_head_stride + 8 * (r + 4));
        }
    }
    sync_128(kLoaderBarrier);
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
        const int h = (tid >> 2) + 32 * k;
        if (h >= N) break;
        uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w}, w[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u[e] = rope_turn(u[e], turn[4 * r + e]);
                w[e] = rope_turn(w[e], turn[4 * r + 16 + e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 c0 = turn[8 * r + 2 * e], c1 = turn[8 * r + 2 * e + 1];
                const float u0 = bf_lo(u[e]), u1 = bf_hi(u[e]), w0 = bf_lo(w[e]), w1 = bf_hi(w[e]);
                u[e] = bf_pack(turn_first(u0, w0, c0), turn_first(u1, w1, c1));
                w[e] = bf_pack(turn_second(u0, w0, c0), turn_second(u1, w1, c1));
            }
        }
        *q_at(h, r) = make_uint4(u[0], u[1], u[2], u[3]);
        *q_at(h, r + 4) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

}  // namespace

// The kernel on pairs of CTAs, for two head groups (latent_decode_pair.cu).  map: pages, latent queries, positional queries, pages'
// halves of the latent part; args: decode_args, whose `groups` may come back smaller (what the device holds at a time).
int latent_decode_pairs(const CUtensorMap (&map)[4], void* args, void* stream);
