// Absorbed latent attention of one query token per block for more than 64 heads: pairs of CTAs (clusters of two, tcgen05
// cta_group::2), each CTA with half of the heads.
//
// Why pairs.  With 64 heads to a CTA the one-CTA kernel (latent_decode.cu) is bound by shared memory: S^T and O^T of a tile of
// 64 tokens read 144 and 96 KB of operands beside the 74 KB that arrive, 2500 cycles at 128 bytes each, and two CTAs do that for
// the same tokens.  Here the heads are on the M side and one instruction drives both tensor cores:
//     S = Q K^T        M = 2 x 64 heads, N = 64 tokens: each CTA stages the rows of 32 tokens, all elements
//     O += P C         M = 2 x 64 heads, N = up to 256 latent elements, K = tokens: each CTA stages all 64 tokens' rows of half of
//                      the latent elements (their positional part is not needed)
// so that each operand is read once for both CTAs' heads: 108 + 48 KB and 70 KB that arrive, 1750 cycles.  The 64 rows of a CTA lie
// in lanes 0-63 of its tensor memory with the first half of an instruction's columns and in lanes 64-127 with the second: scores
// take 32 columns, outputs latent_dim / 2, lanes below 64 holding the first half of the latent elements.
//
// Measured (128 heads, latent parts of 512): one block of 131072 tokens, 151 MB and 36.5 GFLOP, 54.6 us in a row, 55.5 to 62 by single
// calls (65 with a one-CTA group per 64 heads); a step of 16 blocks of 8192 tokens 59 us, 60 to 67 (69).  Bound by the chain within a
// tile of 64 tokens, 2180 cycles where the operands take 1750: scores, softmax and outputs alternate over two tiles in shared memory,
// beside 74 KB of queries.  Arrivals in the leader at cluster scope (release.cluster) cost over 1000 cycles each; CTA-scope ones order
// what these barriers hand over, since data goes between the CTAs through the tensor cores and copies alone.
//
// Shares, segments, partials and the joining kernel are those of latent_decode.cu (a pair is a group, a CTA a head group).
// Per CTA: warps 0-7 softmax and epilogue (thread = head, half of the tokens by lane, half of those by warpgroup), 8-11 queries, new
// rows, rows of zeros, 12 TMA producer, 13 and 14 issuers of the score and output products (leader only), 15 segments.
//
// Synchronisation across the pair:
//   - K and Q arrive for both CTAs' use: their copies count on the leader's barriers, which the leader arms.  V arrives on barriers
//     of its own CTA, whose softmax warps look at them before they hand over their weights.
//   - what the products free or complete is committed to both CTAs (multicast commit); what the softmax frees or completes is
//     arrived at in the leader by the warps of both.
// Every wait is bounded; both CTAs run to the cluster barrier at the end whatever gave up.
#include "latent_decode.cuh"

namespace {

constexpr int kHeads = 64;                      // of a CTA
constexpr int kPairStages = 4;

struct __align__(8) PairDecodeBarriers {
    uint64_t k_full[kPairStages];               // leader
    uint64_t k_empty[kPairStages], v_full[kPairStages], v_empty[kPairStages];
    uint64_t s_full[2], pv_done[2];             // committed to both
    uint64_t s_empty[2], p_full[2];             // leader, 16 warps
    uint64_t q_full, o_empty;                   // leader
    uint64_t q_empty, row_ready, row_taken, drain_s, drain_p;
    uint32_t tmem_base;
};
struct PairDecodeShared {
    PairDecodeBarriers bars;
    SegmentRing ring;
    CutShared cut;
    float2 turn[kRopeDim / 2];
    float column[4][kHeads];                    // per quarter of a tile's tokens and head: maxima, sums
    float first[kHeads];
};

template <int L>
struct PairShape {
    static constexpr int kColumns = L / 64 + 1, kHalf = L / 128;             // column blocks of a row, of half of its latent part
    static constexpr uint32_t kPageBytes = kColumns * 2048, kHalfPageBytes = kHalf * 2048, kQBytes = kColumns * kHeads * 128;
    static constexpr uint32_t kKBytes = 2 * kPageBytes, kVBytes = kTilePages * kHalfPageBytes;
    static constexpr int kFixed = (int)(kQBytes + 2 * kPBytes) + (int)sizeof(PairDecodeShared);
    static constexpr int kFit = (kMaxSmem - kFixed) / (int)(kKBytes + kVBytes);
    static constexpr int kStages = kFit < kPairStages ? kFit : kPairStages;
    static constexpr int kSmem = kFixed + kStages * (int)(kKBytes + kVBytes);
    static_assert(kStages >= 2, "two tiles have to fit");
};

__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
// the shared::cluster address of this CTA's `addr` in the leader
__device__ __forceinline__ uint32_t in_leader(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;\n" : "=r"(r) : "r"(addr));
    return r;
}
// Arrival at a barrier of the leader.  What it publishes is tensor memory or shared memory of the arriving warp's own CTA, which the
// leader's products read through the async proxy; the warp's stores have been made visible to that proxy before (tcgen05 and proxy
// fences).  The release is of CTA scope: one of cluster scope waits for all of the warp's memory traffic, 1000 cycles and more in
// every step of the softmax.
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];\n" :: "r"(cluster_addr) : "memory");
}
// Copies whose bytes count on `bar`, a shared::cluster address that may be the leader's.
__device__ __forceinline__ void pair_load_page(uint32_t dst, const CUtensorMap* map, int group, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %3}], [%4];\n"
        :: "r"(dst), "l"(map), "r"(0), "r"(group), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_4d(uint32_t dst, const CUtensorMap* map, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n"
        :: "r"(dst), "l"(map), "r"(0), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const CUtensorMap* map, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n"
        :: "r"(dst), "l"(map), "r"(0), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %6, 0;\n mov.b64 da, {%1, %2};\n mov.b64 db, {%3, %4};\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %5, p;\n}\n"
        :: "r"(d), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
// The pair's products so far, to the barrier at this offset in both CTAs.
__device__ __forceinline__ void commit_both(uint32_t bar) {
    asm volatile("{\n .reg .b16 m;\n mov.b16 m, 3;\n"
                 " tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n}\n"
                 :: "r"(bar) : "memory");
}
__device__ __forceinline__ void commit_leader(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" :: "r"(bar) : "memory");
}
// Whether `x` holds in any of the 256 softmax threads.
__device__ __forceinline__ bool any_of_256(bool x) {
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, 1, 256, p;\n selp.u32 %0, 1, 0, q;\n}\n"
                 : "=r"(r) : "r"((uint32_t)x) : "memory");
    return r != 0;
}
__device__ __forceinline__ void sync_256() { asm volatile("barrier.cta.sync 1, 256;\n" ::: "memory"); }

template <int L>
__global__ void __launch_bounds__(kDecodeThreads, 1)
latent_decode_pair_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap map_half,
                          const __grid_constant__ CUtensorMap map_qc, const __grid_constant__ CUtensorMap map_qr,
                          const __grid_constant__ decode_args a) {
    extern __shared__ __align__(1024) unsigned char gen[];
    using Sh = PairShape<L>;
    constexpr int nc = Sh::kColumns, vc = Sh::kHalf, kStages = Sh::kStages;
    const uint32_t base = smem_u32(gen);
    if (base & 1023u) {              // swizzled tiles would be misread (both CTAs see the same address)
        if (threadIdx.x == 0) atomicCAS(a.t.header, 0, kStatusInvalid);
        return;
    }
    const uint32_t s_k = base, s_v = s_k + kStages * Sh::kKBytes, s_q = s_v + kStages * Sh::kVBytes, s_p = s_q + Sh::kQBytes;
    PairDecodeShared& sm = *reinterpret_cast<PairDecodeShared*>(gen + (s_p + 2 * kPBytes - base));
    PairDecodeBarriers& bars = sm.bars;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int rank = (int)cta_rank(), group = blockIdx.x >> 1;
    const int h0 = rank * a.group_heads, heads = min(a.group_heads, a.H - h0);
    auto bar = [](uint64_t* p) { return smem_u32(p); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar(&bars.k_full[s]), 1);
            mbar_init(bar(&bars.k_empty[s]), 1);
            mbar_init(bar(&bars.v_full[s]), kTilePages);
            mbar_init(bar(&bars.v_empty[s]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&bars.s_full[i]), 1);
            mbar_init(bar(&bars.pv_done[i]), 1);
            mbar_init(bar(&bars.s_empty[i]), 16);
            mbar_init(bar(&bars.p_full[i]), 16);
        }
        mbar_init(bar(&bars.q_full), a.turns ? 9 : 1);      // the leader's arming, and the loader warps of both that turn
        mbar_init(bar(&bars.o_empty), 16);
        mbar_init(bar(&bars.q_empty), 1);
        mbar_init(bar(&bars.row_ready), 1);
        mbar_init(bar(&bars.row_taken), 1);
        mbar_init(bar(&bars.drain_s), 1);
        mbar_init(bar(&bars.drain_p), 1);
        init_ring(sm.ring, 15);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    }
    if (warp == 13) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;\n" :: "r"(smem_u32(&bars.tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    look_ahead(a);
    if (threadIdx.x == 12 * 32) {
        prefetch_map(&map);
        prefetch_map(&map_half);
        prefetch_map(&map_qc);
        prefetch_map(&map_qr);
    }
    cluster_sync_all();      // both CTAs' barriers are there before anything arrives at them from the other side
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    sum_costs(a, sm.cut);
    const uint32_t tmem = bars.tmem_base;
    constexpr uint32_t kColO = 64;             // two score buffers of 32 columns
    bool dead = false;
    int32_t* const status = a.t.header;
    auto wait = [&](uint64_t* p, uint32_t parity) { mbar_wait(bar(p), parity, dead, status, kSpinLimit); };
    auto get_segment = [&](int i) { return take_segment(sm.ring, i, dead, status); };
    auto pages_of = [](const segment& g, int j) {      // pages of the segment's tile j
        return (int)min((int64_t)kTilePages, ((int64_t)g.len - (int64_t)(g.tile0 + j) * kTile + kPage - 1) / kPage);
    };

    if (warp == 15) {
        hand_out(a, sm.cut, sm.ring, group, rank == 0, dead, status);
    } else if (warp == 12) {
        // ------------------------------------------------------------ TMA producer: lanes 0-1 this CTA's pages of K, lanes 4-7 all
        // pages' halves of V
        int it0 = 0, fresh = 0;
        const uint32_t k_full = in_leader(bar(&bars.k_full[0]));
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (g.block < 0) break;
            const bool is_k = lane < 2, is_v = lane >= 4 && lane < 8;
            if (is_k || is_v) {
                const int mine = is_k ? 2 * rank + lane : lane - 4;          // page of a tile
                const int pages = (int)(((int64_t)g.len + kPage - 1) / kPage);
                const bool grows = a.x && (g.tile0 + g.tiles) * (int64_t)kTile >= g.len;    // holds the step's new token
                int at = g.tile0 * kTilePages + mine;
                int page = at < pages ? ld_i32(a.t.page_indices + g.ip + at) : 0;
                for (int j = 0; j < g.tiles && !dead; ++j, at += kTilePages) {
                    const int s = (it0 + j) % kStages, my = page;
                    const uint32_t par = (uint32_t)((it0 + j) / kStages) & 1u;
                    if (j + 1 < g.tiles && at + kTilePages < pages) page = ld_i32(a.t.page_indices + g.ip + at + kTilePages);
                    wait(is_k ? &bars.k_empty[s] : &bars.v_empty[s], par ^ 1u);
                    if (dead) break;
                    if (rank == 0 && lane == 0) mbar_expect_tx(bar(&bars.k_full[s]), pages_of(g, j) * Sh::kPageBytes);
                    if (at >= pages) {
                        if (is_v) mbar_arrive(bar(&bars.v_full[s]));
                        continue;
                    }
                    if (grows && at == pages - 1) {
                        wait(&bars.row_ready, (uint32_t)fresh & 1u);
                        if (dead) break;
                        asm volatile("fence.proxy.async;\n" ::: "memory");
                        if (is_v) mbar_arrive(bar(&bars.row_taken));
                    }
                    if (is_k) {
                        pair_load_page(s_k + s * Sh::kKBytes + lane * Sh::kPageBytes, &map, my * 2, k_full + 8 * s);
                    } else {
                        mbar_expect_tx(bar(&bars.v_full[s]), Sh::kHalfPageBytes);
                        asm volatile(
                            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4}], [%5];\n"
                            :: "r"(s_v + s * Sh::kVBytes + mine * Sh::kHalfPageBytes), "l"(&map_half), "r"(0), "r"(rank * vc), "r"(my * 2),
                               "r"(bar(&bars.v_full[s])) : "memory");
                    }
                }
                if (grows) ++fresh;
            }
            it0 += g.tiles;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
        // After a wait gave up: copies issued last may still be on their way (the peer's K counts on the leader's barriers; the
        // peer cannot leave before the leader reaches the cluster barrier).
        if (__any_sync(0xffffffffu, dead) && lane == 0)
            for (int s = 0; s < kStages; ++s)
                for (uint32_t par = 0; par < 2; ++par) {
                    if (rank == 0) mbar_drain(bar(&bars.k_full[s]), par, kDrainLimit);
                    mbar_drain(bar(&bars.v_full[s]), par, kDrainLimit);
                }
    } else if (warp == 13) {
        // ------------------------------------------------------------ score products, by one lane of the leader
        constexpr uint32_t idesc = instr_desc(128, kTile, false);
        const uint64_t da = smem_desc(s_q, 16, 1024), db = smem_desc(s_k, 16, nc * 1024);
        const uint32_t a_hi = (uint32_t)(da >> 32), b_hi = (uint32_t)(db >> 32), a_lo = (uint32_t)da;
        int it0 = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (g.block < 0) break;
            if (rank == 0 && elect_one()) {
                wait(&bars.q_full, (uint32_t)i & 1u);
                int it = it0;
                for (int j = 0; j < g.tiles && !dead; ++j, ++it) {
                    const int s = it % kStages;
                    wait(&bars.k_full[s], (uint32_t)(it / kStages) & 1u);
                    wait(&bars.s_empty[it & 1], ((uint32_t)(it >> 1) & 1u) ^ 1u);
                    if (dead) break;
                    tc_fence_after();
                    const uint32_t b_lo = (uint32_t)db + (uint32_t)s * (Sh::kKBytes >> 4), d = tmem + (it & 1) * 32;
#pragma unroll
                    for (int k = 0; k < nc * 4; ++k)
                        pair_mma(d, a_lo + ((k >> 2) * (kHeads * 128) + (k & 3) * 32 >> 4), a_hi, b_lo + ((k >> 2) * 1024 + (k & 3) * 32 >> 4), b_hi,
                                 idesc, k != 0);
                    commit_both(bar(&bars.s_full[it & 1]));
                    commit_both(bar(&bars.k_empty[s]));
                }
                if (!dead) commit_both(bar(&bars.q_empty));
            }
            it0 += g.tiles;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
        if (dead && rank == 0 && elect_one()) {      // products queued before may still be running
            commit_leader(bar(&bars.drain_s));
            mbar_drain(bar(&bars.drain_s), 0u, kDrainLimit);
        }
    } else if (warp == 14) {
        // ------------------------------------------------------------ output products, by one lane of the leader
        const uint64_t da = smem_desc(s_p, 16, 1024), db = smem_desc(s_v, 1024, vc * 1024);
        const uint32_t a_hi = (uint32_t)(da >> 32), b_hi = (uint32_t)(db >> 32);
        int it0 = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (g.block < 0) break;
            if (rank == 0 && elect_one()) {
                if (i > 0) wait(&bars.o_empty, (uint32_t)(i - 1) & 1u);
                int it = it0;
                for (int j = 0; j < g.tiles && !dead; ++j, ++it) {
                    const int s = it % kStages, pages = pages_of(g, j);
                    wait(&bars.p_full[it & 1], (uint32_t)(it >> 1) & 1u);
                    if (dead) break;
                    tc_fence_after();
                    const uint32_t a_lo = (uint32_t)da + (uint32_t)(it & 1) * (kPBytes >> 4), b_lo = (uint32_t)db + (uint32_t)s * (Sh::kVBytes >> 4);
#pragma unroll
                    for (int p = 0; p < kTilePages; ++p) {
                        if (p < pages) {
#pragma unroll
                            for (int v = 0; v < vc; v += 2)      // up to two column blocks of each CTA per instruction
                                pair_mma(tmem + kColO + v * 64, a_lo + (p * 32 >> 4), a_hi, b_lo + (p * Sh::kHalfPageBytes + v * 1024 >> 4), b_hi,
                                         vc - v >= 2 ? instr_desc(128, 256, true) : instr_desc(128, 128, true), p != 0 || j != 0);
                        }
                    }
                    commit_both(bar(&bars.v_empty[s]));
                    commit_both(bar(&bars.pv_done[it & 1]));
                }
            }
            it0 += g.tiles;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
        if (dead && rank == 0 && elect_one()) {
            commit_leader(bar(&bars.drain_p));
            mbar_drain(bar(&bars.drain_p), 0u, kDrainLimit);
        }
    } else if (warp >= 8) {
        // ------------------------------------------------------------ queries, a step's new row, rows of zeros
        const int tid = threadIdx.x - 256;
        auto q_at = [&](int h, int p) {                // where piece p of head h's positional part lies (swizzled)
            return reinterpret_cast<uint4*>(gen + (s_q - base) + (nc - 1) * (kHeads * 128) + h * 128 + ((p ^ (h & 7)) << 4));
        };
        const uint32_t q_full = in_leader(bar(&bars.q_full));
        int fresh = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (any_of_128(kLoaderBarrier, g.block < 0)) break;
            const int position = (a.first ? ld_i32(a.first + g.block) : 0) + g.len - 1;
            if (i > 0) wait(&bars.q_empty, (uint32_t)(i - 1) & 1u);
            if (warp == 9) {
                if (lane == 0 && !dead) {
                    constexpr uint32_t kTurned = kHeads * 128;
                    if (rank == 0) mbar_expect_tx(bar(&bars.q_full), 2 * (Sh::kQBytes - (a.turns ? kTurned : 0)));
                    pair_load_4d(s_q, &map_qc, h0, 0, g.block, q_full);
                    if (!a.turns) pair_load_3d(s_q + (nc - 1) * kTurned, &map_qr, h0, g.block, q_full);
                }
                if (a.turns) sm.turn[lane] = rope_cos_sin(ld_u64(a.turns + lane), position, a.amplitude);
                __syncwarp();
            }
            if (a.turns) {
                turn_queries<kHeads>(a, g.block, h0, heads, tid, sm.turn, q_at);
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_cluster(q_full);
            }
            if (warp == 8 && a.x && (g.tile0 + g.tiles) * (int64_t)kTile >= g.len) {
                // Both CTAs make the row, each for its own copies.  (K of the last growing segment has been loaded: its scores are
                // through, or these queries could not have been stored; V may lag behind.)
                if (fresh > 0) wait(&bars.row_taken, (uint32_t)(fresh - 1) & 1u);
                put_new_row<L>(a.x + g.block * a.x_row, new_row_of(a), position, slot_of<L>(a, g), lane);
                asm volatile("fence.proxy.async;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars.row_ready));
                ++fresh;
            }
        }
        keep_books(a, tid);
    } else {
        // ------------------------------------------------------------ softmax and epilogue
        // This thread: head `head` (TMEM lane row + 64 * half), tokens 32 half + 16 part .. + 15 of a tile.
        const int part = warp >> 2, row = (warp & 3) * 32 + lane, half = row >> 6, head = row & 63, quarter = 2 * half + part;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int token = 16 * quarter;
        const uint32_t s_empty = in_leader(bar(&bars.s_empty[0])), p_full = in_leader(bar(&bars.p_full[0])), o_empty = in_leader(bar(&bars.o_empty));
        constexpr int kOut = L / 4;            // latent elements of this thread's share of the output
        const uint32_t t_o = tmem + lanes + kColO + part * kOut;
        int it = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (any_of_256(g.block < 0)) break;
            float m = kLowest, l = 0.f;
            for (int j = 0; j < g.tiles; ++j, ++it) {
                const int b = it & 1, stage = it % kStages;
                const int valid = (int)min((int64_t)kTile, (int64_t)g.len - (int64_t)(g.tile0 + j) * kTile);
                wait(&bars.s_full[b], (uint32_t)(it >> 1) & 1u);
                tc_fence_after();
                float s[16];
                tc_ld16(tmem + lanes + b * 32 + 16 * part, s);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_cluster(s_empty + 8 * b);
                // V of the tile has landed here (and, by this warp's arrival below, is the products' to read)
                wait(&bars.v_full[stage], (uint32_t)(it / kStages) & 1u);
                if (valid < kTile) {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (token + e >= valid) s[e] = -INFINITY;
                    // rows behind the length hold anything, and their weights of zero would not silence an infinity or a NaN
                    for (int e = threadIdx.x; e < (kTile - valid) * (vc * 8) && !dead; e += 256) {
                        const int t = valid + e / (vc * 8), p = e % (vc * 8);
                        *reinterpret_cast<uint4*>(gen + (s_v - base) + stage * Sh::kVBytes + (t >> 3) * (vc * 1024) + (p >> 3) * 1024 + (t & 7) * 128 +
                                                  ((p & 7) << 4)) = make_uint4(0, 0, 0, 0);
                    }
                }
                if (j == 0) {              // the first reference, as in the one-CTA kernel
                    if (quarter == 0) sm.first[head] = s[0];
                    sync_256();
                    const float x = fmaf(sm.first[head], a.scale_log2, kFirstMargin);
                    m = fabsf(x) < 1e38f ? x : kLowest;
                }
                bool high = false;
#pragma unroll
                for (int e = 0; e < 16; ++e) high |= fmaf(s[e], a.scale_log2, -m) > 8.f;
                if (any_of_256(high || dead)) {
                    if (any_of_256(dead)) { dead = true; break; }
                    float x = s[0];
#pragma unroll
                    for (int e = 1; e < 16; ++e) x = fmaxf(x, s[e]);
                    sm.column[quarter][head] = x;
                    sync_256();
                    x = a.scale_log2 * fmaxf(fmaxf(sm.column[0][head], sm.column[1][head]), fmaxf(sm.column[2][head], sm.column[3][head]));
                    float f = 1.f;
                    if (x - m > 8.f) {
                        f = exp2f(m - x);
                        m = x;
                    }
                    l *= f;
                    sync_256();            // everyone has read the maxima
                    if (j > 0) {
                        wait(&bars.pv_done[b ^ 1], (uint32_t)((it - 1) >> 1) & 1u);
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < kOut; c += 8) {
                            float v[8];
                            tc_ld8(t_o + c, v);
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = mul_keep(v[e], f);
                            tc_st8(t_o + c, v);
                        }
                        tc_wait_st();
                    }
                }
                // the weights' buffer is free once the products of the tile before last have run
                if (it > 1) wait(&bars.pv_done[b], (uint32_t)((it - 2) >> 1) & 1u);
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    w[e >> 1] = bf_pack(exp2f(fmaf(s[e], a.scale_log2, -m)), exp2f(fmaf(s[e + 1], a.scale_log2, -m)));
                    l += bf_lo(w[e >> 1]) + bf_hi(w[e >> 1]);
                }
                unsigned char* const p = gen + (s_p - base) + b * kPBytes + head * 128;
                *reinterpret_cast<uint4*>(p + (((2 * quarter) ^ (head & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(p + (((2 * quarter + 1) ^ (head & 7)) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_cluster(p_full + 8 * b);
            }
            if (any_of_256(dead)) break;
            // ---- the segment's end: sums over the tokens, then the outputs or the partial
            sm.column[quarter][head] = l;
            wait(&bars.pv_done[(it - 1) & 1], (uint32_t)((it - 1) >> 1) & 1u);
            dead = any_of_256(dead);
            tc_fence_after();
            l = (sm.column[0][head] + sm.column[1][head]) + (sm.column[2][head] + sm.column[3][head]);
            const bool mine = head < heads && !dead;
            const int64_t at = ((int64_t)g.slot * 2 + rank) * 64 + head;
            const int dim = half * (L / 2) + part * kOut;
            if (g.slot >= 0) {
                if (quarter == 0 && mine) a.part_ml[at] = make_float2(m, l);
#pragma unroll 1
                for (int c = 0; c < kOut; c += 8) {
                    float v[8];
                    tc_ld8(t_o + c, v);
                    if (mine) {            // a whole sector per lane
                        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n"
                                     :: "l"(a.part_o + at * L + dim + c), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
                                        "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])),
                                        "r"(__float_as_uint(v[7])) : "memory");
                    }
                }
            } else {
                const float f = 1.f / l;
                __nv_bfloat16* o = (__nv_bfloat16*)a.io.o + g.block * a.io.o_block_stride + (h0 + head) * a.io.o_head_stride + dim;
#pragma unroll 1
                for (int c = 0; c < kOut; c += 8) {
                    float v[8];
                    tc_ld8(t_o + c, v);
                    if (mine)
                        *reinterpret_cast<uint4*>(o + c) =
                            make_uint4(bf_pack(mul_keep(v[0], f), mul_keep(v[1], f)), bf_pack(mul_keep(v[2], f), mul_keep(v[3], f)),
                                       bf_pack(mul_keep(v[4], f), mul_keep(v[5], f)), bf_pack(mul_keep(v[6], f), mul_keep(v[7], f)));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_cluster(o_empty);
        }
    }

    // Neither CTA may leave, or free its tensor memory, while the other may still read its shared memory, write its barriers or run
    // products over its tensor memory.
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 13) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;\n" :: "r"(tmem) : "memory");
    }
}

// Makes the kernel ready on the current device and says how many pairs it holds at a time; 0 if that cannot be found out.
template <int L>
int pairs_held() {
    static std::atomic<int> known[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        (void)cudaGetLastError();
        return 0;
    }
    int n = known[dev].load(std::memory_order_relaxed);
    if (n) return n;
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    lc.gridDim = dim3(kSms);
    lc.blockDim = dim3(kDecodeThreads);
    lc.dynamicSmemBytes = PairShape<L>::kSmem;
    lc.attrs = attr;
    lc.numAttrs = 1;
    if (cudaFuncSetAttribute(latent_decode_pair_kernel<L>, cudaFuncAttributeMaxDynamicSharedMemorySize, PairShape<L>::kSmem) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, latent_decode_pair_kernel<L>, &lc) != cudaSuccess || n < 1) {
        (void)cudaGetLastError();
        return 0;
    }
    known[dev].store(n, std::memory_order_relaxed);
    return n;
}

template <int L>
int launch(const CUtensorMap (&map)[4], decode_args& a, cudaStream_t st) {
    const int held = pairs_held<L>();
    if (held < 1) return CPA_ECUDA;
    a.groups = std::min(a.groups, held);          // one wave
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3((unsigned)a.groups * 2);
    lc.blockDim = dim3(kDecodeThreads);
    lc.dynamicSmemBytes = PairShape<L>::kSmem;
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 2;
    if (cudaLaunchKernelEx(&lc, latent_decode_pair_kernel<L>, map[0], map[3], map[1], map[2], a) != cudaSuccess) {
        (void)cudaGetLastError();
        return CPA_ECUDA;
    }
    return CPA_OK;
}

}  // namespace

// map: pages, latent queries, positional queries, pages' halves.  a.groups may come back smaller (what the device holds at a time).
int latent_decode_pairs(const CUtensorMap (&map)[4], void* args, void* stream) {
    decode_args& a = *static_cast<decode_args*>(args);
    cudaStream_t st = (cudaStream_t)stream;
    switch (a.L) {
        case 128: return launch<128>(map, a, st);
        case 256: return launch<256>(map, a, st);
        case 384: return launch<384>(map, a, st);
        default: return launch<512>(map, a, st);
    }
}
