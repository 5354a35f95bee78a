// Absorbed latent attention of one query token per block over the paged latent cache, on the tensor cores.
//
//     S^T = K Q^T            [tokens, heads]     K: 64 rows of the cache, all latent_dim + 64 elements
//     P^T = exp2(S^T - m)    m: a running reference of each head's maximum
//     O^T += C^T P^T         [latent elements, heads]     C: the same 64 rows without their positional part
//
// The rows are staged once (TMA, one copy per page) and serve both products: as the K-major operand of the first and the
// MN-major operand of the second.  Tokens and latent elements are on the M side, so 16, 32 or 64 heads fill N without waste, and
// O^T (latent_dim / 128 accumulators of 128 lanes x heads columns) leaves room in tensor memory for two score buffers at 64
// heads; with the heads on the M side the 512-wide outputs of 128 rows would take all of it.  More than 64 heads go to pairs of
// CTAs (latent_decode_pair.cu).
//
// A CTA owns an equal share of all blocks' 64-token tiles, cut on the device from the lengths; a block that is cut leaves
// partial sums in the workspace, which a second kernel joins.  Sixteen warps with fixed roles:
//   0-3   softmax of the first half of the heads: warp w holds tokens 16 w .. 16 w + 15 of a tile in the fragment layout of a
//         16-lane TMEM load; epilogue of the same heads
//   4-7   the same for the second half
//   8-11  queries of the next segment into shared memory (turned, if asked for), a step's new row; rows of zeros
//   12    TMA producer, one lane per page of a tile
//   13    issuer of the score products; owner of the tensor memory
//   14    issuer of the output products (a warp of its own, so that neither product waits behind the other's operands)
//   15    walks the blocks and hands out the segments (block, first tile, tiles)
// The reference m of a head stays as long as no score passes it by more than 2^8 (what it is cancels in the division); the
// four warps of a half learn of that by one barrier with an OR, so a tile usually costs no exchange of maxima at all.
//
// Measured (latent parts of 512, caches larger than L2): 64 heads over 32 blocks of 1024..8192 tokens, 195 MB, 57 us (3.4 TB/s) in a row;
// 16 heads over 192 blocks of 512..1024 with a step's new rows, 175 MB, 46 us (3.8 TB/s); 16 heads over 4 blocks of up to 288
// tokens 8.8 us.  What bounds it: the stream of pages runs at 5.8 TB/s once it runs (a tile of 74 KB every 3550 cycles at 64
// heads, 3150 at 16: memory's latency under that load, 3400 cycles, and the chain of a tile, twice over in two stages; beside 74 KB
// of queries no third tile fits, and the operands of both products take 2500 cycles of shared memory's time as it is).  Around it:
// 3 us from the start to the first copy (cut, segment, page list: loads that depend on one another), 3.5 us for the partials
// (128 KB from every CTA at 64 heads, 5.5 TB/s), 3.5 us from the median CTA to the last, 1 us to the join and 5 to 7.5 us in it.
// Looking ahead with L2 prefetches of pages cost 5 to 15 us (the copies queue behind them).
//
// Every mbarrier wait is bounded: when one gives up the CTA records it in the status word, stops waiting, still frees its
// tensor memory and returns.
#include "latent_decode.cuh"

namespace {

constexpr int kMaxDecodeStages = 6;

struct __align__(8) DecodeBarriers {
    uint64_t kv_full[kMaxDecodeStages], kv_empty[kMaxDecodeStages][kTilePages];
    uint64_t s_full[2], s_empty[2], p_full, pv_done, q_full, q_empty, o_empty, row_ready, drain_s, drain_p;
    uint32_t tmem_base;
};

template <int N>
struct DecodeShared {
    DecodeBarriers bars;
    SegmentRing ring;
    CutShared cut;
    float2 turn[kRopeDim / 2];
    float column[8][N / 2];           // per warp and head: maxima, sums
    float factor[N];
};

template <int L, int N>
struct DecodeShape {
    static constexpr int kColumns = L / 64 + 1;                              // 64-element column blocks of a row
    static constexpr uint32_t kPageBytes = kColumns * 2048, kQBytes = kColumns * N * 128;
    static constexpr int kFixed = (int)(kQBytes + kPBytes) + (int)sizeof(DecodeShared<N>);
    static constexpr int kFit = (kMaxSmem - kFixed) / (int)(kTilePages * kPageBytes);
    static constexpr int kStages = kFit < kMaxDecodeStages ? kFit : kMaxDecodeStages;
    static constexpr int kSmem = kFixed + kStages * kTilePages * (int)kPageBytes;
    static_assert(kStages >= 2, "two tiles have to fit");
    static_assert(2 * N + L / 128 * N <= 512, "tensor memory");
};

// ---------------------------------------------------------------- PTX
// By one thread; descriptors as halves, of which the lower one holds the address.
__device__ __forceinline__ void tc_mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                          uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %6, 0;\n mov.b64 da, {%1, %2};\n mov.b64 db, {%3, %4};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %5, p;\n}\n"
        :: "r"(d_tmem), "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_commit_one(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" :: "r"(bar) : "memory");
}
// Columns of 16 lanes in fragment layout: per 8 columns four words, of lane / 4 (words 0, 1) and lane / 4 + 8 (words 2, 3),
// columns 2 (lane % 4) and the next.
template <int N> __device__ __forceinline__ void tc_ld_frag(uint32_t taddr, float (&v)[N / 2]);
template <> __device__ __forceinline__ void tc_ld_frag<8>(uint32_t taddr, float (&v)[4]) {
    uint32_t r[4];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
template <> __device__ __forceinline__ void tc_ld_frag<16>(uint32_t taddr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
template <> __device__ __forceinline__ void tc_ld_frag<32>(uint32_t taddr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(taddr) : "memory");
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
template <int L, int N>
__global__ void __launch_bounds__(kDecodeThreads, 1)
latent_decode_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap map_qc,
                     const __grid_constant__ CUtensorMap map_qr, const __grid_constant__ decode_args a) {
    extern __shared__ __align__(1024) unsigned char gen[];       // (the kernel has no other shared memory, so this is its start)
    const uint32_t base = smem_u32(gen);
    if (base & 1023u) {              // swizzled tiles would be misread
        if (threadIdx.x == 0) atomicCAS(a.t.header, 0, kStatusInvalid);
        return;
    }
    using Sh = DecodeShape<L, N>;
    constexpr int nc = Sh::kColumns, nm = L / 128;            // column blocks of a row, 128-element blocks of the output
    constexpr int kStages = Sh::kStages;
    constexpr uint32_t page_bytes = Sh::kPageBytes, kTileBytes64 = kTilePages * page_bytes;
    const uint32_t s_kv = base, s_q = s_kv + kStages * kTileBytes64, s_p = s_q + Sh::kQBytes;
    DecodeShared<N>& sm = *reinterpret_cast<DecodeShared<N>*>(gen + (s_p + kPBytes - base));
    DecodeBarriers& bars = sm.bars;
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int group = blockIdx.x, heads = a.H;
    auto bar = [](uint64_t* p) { return smem_u32(p); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(bar(&bars.kv_full[s]), kTilePages);
            for (int p = 0; p < kTilePages; ++p) mbar_init(bar(&bars.kv_empty[s][p]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&bars.s_full[i]), 1);
            mbar_init(bar(&bars.s_empty[i]), 8);
        }
        mbar_init(bar(&bars.p_full), 8);
        mbar_init(bar(&bars.pv_done), 1);
        mbar_init(bar(&bars.q_full), a.turns ? 5 : 4);      // warps 8-11, and the copies beside what warp 9 turns
        mbar_init(bar(&bars.q_empty), 1);
        mbar_init(bar(&bars.o_empty), 8);
        mbar_init(bar(&bars.row_ready), 1);
        mbar_init(bar(&bars.drain_s), 1);
        mbar_init(bar(&bars.drain_p), 1);
        init_ring(sm.ring, 15);                   // every warp but the one that hands out
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    }
    if (warp == 13) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" :: "r"(smem_u32(&bars.tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    look_ahead(a);
    if (threadIdx.x == 12 * 32) {
        prefetch_map(&map);
        prefetch_map(&map_qc);
        prefetch_map(&map_qr);
    }
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    sum_costs(a, sm.cut);
    const uint32_t tmem = bars.tmem_base;
    constexpr uint32_t kColO = 2 * N;
    bool dead = false;
    int32_t* const status = a.t.header;
    auto wait = [&](uint64_t* p, uint32_t parity) { mbar_wait(bar(p), parity, dead, status, kSpinLimit); };
    auto get_segment = [&](int i) { return take_segment(sm.ring, i, dead, status); };

    if (warp == 15) {
        hand_out(a, sm.cut, sm.ring, group, true, dead, status);
    } else if (warp == 12) {
        // ------------------------------------------------------------ TMA producer, a lane per page
        int it = 0, fresh = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (g.block < 0) break;
            if (lane < kTilePages) {
                const int pages = (int)(((int64_t)g.len + kPage - 1) / kPage);
                int at = g.tile0 * kTilePages + lane;
                int page = at < pages ? ld_i32(a.t.page_indices + g.ip + at) : 0;
                const bool grows = a.x && (g.tile0 + g.tiles) * (int64_t)kTile >= g.len;    // holds the step's new token
                for (int j = 0; j < g.tiles && !dead; ++j, at += kTilePages) {
                    const int s = (it + j) % kStages, my = page;
                    const uint32_t par = (uint32_t)((it + j) / kStages) & 1u;
                    if (j + 1 < g.tiles && at + kTilePages < pages) page = ld_i32(a.t.page_indices + g.ip + at + kTilePages);
                    wait(&bars.kv_empty[s][lane], par ^ 1u);
                    if (dead) break;
                    if (at >= pages) {
                        mbar_arrive(bar(&bars.kv_full[s]));
                        continue;
                    }
                    if (grows && at == pages - 1) {
                        wait(&bars.row_ready, (uint32_t)fresh & 1u);
                        if (dead) break;
                        asm volatile("fence.proxy.async;\n" ::: "memory");
                    }
                    mbar_expect_tx(bar(&bars.kv_full[s]), page_bytes);
                    tma_load_page(s_kv + (s * kTilePages + lane) * page_bytes, &map, my * 2, bar(&bars.kv_full[s]));
                }
                if (grows) ++fresh;
            }
            it += g.tiles;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
        // After a wait gave up: copies issued last may still be on their way into this CTA's shared memory.
        if (__any_sync(0xffffffffu, dead) && lane == 0)
            for (int s = 0; s < kStages; ++s)
                for (uint32_t par = 0; par < 2; ++par) mbar_drain(bar(&bars.kv_full[s]), par, kDrainLimit);
    } else if (warp == 13) {
        // ------------------------------------------------------------ score products, by one lane
        constexpr uint32_t idesc = instr_desc(kTile, N, false);
        const uint64_t da = smem_desc(s_kv, 16, nc * 1024), db = smem_desc(s_q, 16, 1024);
        const uint32_t a_hi = (uint32_t)(da >> 32), b_hi = (uint32_t)(db >> 32), b_lo = (uint32_t)db;
        int it0 = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (g.block < 0) break;
            if (elect_one()) {
                int it = it0;
                wait(&bars.q_full, (uint32_t)i & 1u);
                for (int j = 0; j < g.tiles && !dead; ++j, ++it) {
                    const int s = it % kStages;
                    wait(&bars.kv_full[s], (uint32_t)(it / kStages) & 1u);
                    wait(&bars.s_empty[it & 1], ((uint32_t)(it >> 1) & 1u) ^ 1u);
                    if (dead) break;
                    tc_fence_after();
                    const uint32_t a_lo = (uint32_t)da + (uint32_t)s * (kTileBytes64 >> 4), d = tmem + (it & 1) * N;
#pragma unroll
                    for (int k = 0; k < nc * 4; ++k)
                        tc_mma_ss(d, a_lo + ((k >> 2) * 1024 + (k & 3) * 32 >> 4), a_hi, b_lo + ((k >> 2) * (N * 128) + (k & 3) * 32 >> 4), b_hi,
                                  idesc, k != 0);
                    tc_commit_one(bar(&bars.s_full[it & 1]));
                }
                if (!dead) tc_commit_one(bar(&bars.q_empty));
            }
            it0 += g.tiles;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
        if (dead && elect_one()) {      // products queued before may still be running; tensor memory is not freed under them
            tc_commit_one(bar(&bars.drain_s));
            mbar_drain(bar(&bars.drain_s), 0u, kDrainLimit);
        }
    } else if (warp == 14) {
        // ------------------------------------------------------------ output products, by one lane
        constexpr uint32_t idesc = instr_desc(128, N, true) | (1u << 15);       // both operands MN-major
        const uint64_t da = smem_desc(s_kv, 1024, nc * 1024), db = smem_desc(s_p, 16, 1024);
        const uint32_t a_hi = (uint32_t)(da >> 32), b_hi = (uint32_t)(db >> 32), b_lo = (uint32_t)db;
        int it0 = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (g.block < 0) break;
            if (elect_one()) {
                int it = it0;
                if (i > 0) wait(&bars.o_empty, (uint32_t)(i - 1) & 1u);
                for (int j = 0; j < g.tiles && !dead; ++j, ++it) {
                    const int s = it % kStages;
                    const int pages = (int)min((int64_t)kTilePages, ((int64_t)g.len - (int64_t)(g.tile0 + j) * kTile + kPage - 1) / kPage);
                    wait(&bars.p_full, (uint32_t)it & 1u);
                    if (dead) break;
                    tc_fence_after();
                    const uint32_t a_lo = (uint32_t)da + (uint32_t)s * (kTileBytes64 >> 4);
#pragma unroll
                    for (int p = 0; p < kTilePages; ++p) {
                        if (p < pages) {
#pragma unroll
                            for (int m = 0; m < nm; ++m)
                                tc_mma_ss(tmem + kColO + m * N, a_lo + (p * page_bytes + m * 2048 >> 4), a_hi, b_lo + (p * 2048 >> 4), b_hi, idesc,
                                          p != 0 || j != 0);
                        }
                        tc_commit_one(bar(&bars.kv_empty[s][p]));
                    }
                    tc_commit_one(bar(&bars.pv_done));
                }
            }
            it0 += g.tiles;
            dead = __any_sync(0xffffffffu, dead);
            if (dead) break;
        }
        if (dead && elect_one()) {
            tc_commit_one(bar(&bars.drain_p));
            mbar_drain(bar(&bars.drain_p), 0u, kDrainLimit);
        }
    } else if (warp >= 8) {
        // ------------------------------------------------------------ queries, a step's new row, rows of zeros
        // (loops are kept short: what a launch runs once or twice costs the fetching of its instructions)
        const int tid = threadIdx.x - 256;
        auto q_at = [&](int h, int p) {                // where piece p of head h's positional part lies (swizzled)
            return reinterpret_cast<uint4*>(gen + (s_q - base) + (nc - 1) * (N * 128) + h * 128 + ((p ^ (h & 7)) << 4));
        };
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (any_of_128(kLoaderBarrier, g.block < 0)) break;
            const int position = (a.first ? ld_i32(a.first + g.block) : 0) + g.len - 1;
            if (i > 0) wait(&bars.q_empty, (uint32_t)(i - 1) & 1u);
            if (warp == 9) {
                // the latent parts, and the positional ones that do not turn; heads behind the last are filled with zeros
                if (lane == 0 && !dead) {
                    mbar_expect_tx(bar(&bars.q_full), Sh::kQBytes - (a.turns ? N * 128 : 0));
                    tma_load_q(s_q, &map_qc, 0, g.block, bar(&bars.q_full));
                    if (!a.turns) tma_load_3d(s_q + (nc - 1) * (N * 128), &map_qr, 0, 0, g.block, bar(&bars.q_full));
                }
                if (a.turns) sm.turn[lane] = rope_cos_sin(ld_u64(a.turns + lane), position, a.amplitude);
                __syncwarp();
            }
            if (a.turns) {
                turn_queries<N>(a, g.block, 0, heads, tid, sm.turn, q_at);
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                __syncwarp();
            }
            if (lane == 0 && warp != 9) mbar_arrive(bar(&bars.q_full));
            if (lane == 0 && warp == 9 && a.turns) mbar_arrive(bar(&bars.q_full));
            // (the last growing segment's row has been loaded: its scores are through, or these queries could not have been stored)
            if (warp == 8 && a.x && (g.tile0 + g.tiles) * (int64_t)kTile >= g.len) {
                put_new_row<L>(a.x + g.block * a.x_row, new_row_of(a), position, slot_of<L>(a, g), lane);
                asm volatile("fence.proxy.async;\n" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars.row_ready));
            }
        }
        keep_books(a, tid);
    } else {
        // ------------------------------------------------------------ softmax and epilogue
        constexpr int NH = N / 2, J = NH / 8;  // heads of a half; groups of eight, of which this thread has two heads and two tokens
        const int which = warp >> 2, quarter = warp & 3, id = 1 + which, h1 = which * NH;
        const int token = 16 * quarter + (lane >> 2), col = 2 * (lane & 3);
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        float (*column)[NH] = sm.column + 4 * which;
        float* factor = sm.factor + h1;
        int it = 0;
        for (int i = 0;; ++i) {
            const segment g = get_segment(i);
            if (any_of_128(id, g.block < 0)) break;
            float m[2 * J], l[2 * J];
#pragma unroll
            for (int k = 0; k < 2 * J; ++k) { m[k] = kLowest; l[k] = 0.f; }
            for (int j = 0; j < g.tiles; ++j, ++it) {
                const int valid = (int)min((int64_t)kTile, (int64_t)g.len - (int64_t)(g.tile0 + j) * kTile);
                wait(&bars.s_full[it & 1], (uint32_t)(it >> 1) & 1u);
                tc_fence_after();
                float s[4 * J];
                tc_ld_frag<NH>(tmem + lanes + (it & 1) * N + h1, s);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars.s_empty[it & 1]));
                if (valid < kTile) {
#pragma unroll
                    for (int k = 0; k < J; ++k) {
                        if (token >= valid) s[4 * k] = s[4 * k + 1] = -INFINITY;
                        if (token + 8 >= valid) s[4 * k + 2] = s[4 * k + 3] = -INFINITY;
                    }
                    // rows behind the length hold anything, and their weights of zero would not silence an infinity or a NaN
                    constexpr int row16 = L / 8;
                    const int stage = it % kStages;
                    for (int e = threadIdx.x; e < (kTile - valid) * row16; e += 256) {
                        const int t = valid + e / row16, p = e % row16;
                        *reinterpret_cast<uint4*>(gen + stage * kTileBytes64 + (t >> 3) * (nc * 1024) + (p >> 3) * 1024 + (t & 7) * 128 +
                                                  ((p & 7) << 4)) = make_uint4(0, 0, 0, 0);
                    }
                }
                if (j == 0) {
                    // The first reference: the first token's score and a margin (with N(0, 2^2) scores the largest of a long block
                    // is then mostly within 2^8 of it); the true maximum takes over where it is not.
                    if (quarter == 0 && lane < 4)
#pragma unroll
                        for (int k = 0; k < J; ++k)
#pragma unroll
                            for (int e = 0; e < 2; ++e) factor[8 * k + col + e] = s[4 * k + e];
                    sync_128(id);
#pragma unroll
                    for (int k = 0; k < J; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float x = fmaf(factor[8 * k + col + e], a.scale_log2, kFirstMargin);
                            m[2 * k + e] = fabsf(x) < 1e38f ? x : kLowest;
                        }
                }
                bool high = false;
#pragma unroll
                for (int k = 0; k < J; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) high |= fmaf(s[4 * k + e], a.scale_log2, -m[2 * k + (e & 1)]) > 8.f;
                if (any_of_128(id, high || dead)) {
                    if (any_of_128(id, dead)) { dead = true; break; }
                    // some score is far above its head's reference: new references, and what was summed so far is scaled to them
#pragma unroll
                    for (int k = 0; k < J; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float x = fmaxf(s[4 * k + e], s[4 * k + e + 2]);
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
                            if (lane < 4) column[quarter][8 * k + col + e] = x;
                        }
                    sync_128(id);
#pragma unroll
                    for (int k = 0; k < J; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int h = 8 * k + col + e;
                            const float x = a.scale_log2 * fmaxf(fmaxf(column[0][h], column[1][h]), fmaxf(column[2][h], column[3][h]));
                            float& r = m[2 * k + e];
                            float f = 1.f;
                            if (x - r > 8.f) {
                                f = exp2f(r - x);
                                r = x;
                            }
                            l[2 * k + e] *= f;
                            if (quarter == 0 && lane < 4) factor[h] = f;
                        }
                    sync_128(id);
                    if (j > 0) {
                        wait(&bars.pv_done, (uint32_t)(it - 1) & 1u);
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < nm * NH; c += 8) {
                            const uint32_t at = tmem + lanes + kColO + c / NH * N + h1 + c % NH;
                            float v[8];
                            tc_ld8(at, v);
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = mul_keep(v[e], factor[c % NH + e]);
                            tc_st8(at, v);
                        }
                        tc_wait_st();
                    }
                }
                // the weights' buffer is free once the previous tile's products have run
                if (it > 0) wait(&bars.pv_done, (uint32_t)(it - 1) & 1u);
#pragma unroll
                for (int k = 0; k < J; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {       // token, token + 8
                        const uint32_t w = bf_pack(exp2f(fmaf(s[4 * k + 2 * e], a.scale_log2, -m[2 * k])),
                                                   exp2f(fmaf(s[4 * k + 2 * e + 1], a.scale_log2, -m[2 * k + 1])));
                        l[2 * k] += bf_lo(w);
                        l[2 * k + 1] += bf_hi(w);
                        const int t = token + 8 * e;
                        *reinterpret_cast<uint32_t*>(gen + (s_p - base) + t * 128 + (((k + which * J) ^ (t & 7)) << 4) + 2 * col) = w;
                    }
                asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars.p_full));
            }
            if (any_of_128(id, dead)) break;
            // ---- the segment's end: sums over the tokens, then the outputs or the partial
#pragma unroll
            for (int k = 0; k < 2 * J; ++k) {
                float x = l[k];
                x += __shfl_xor_sync(0xffffffffu, x, 4);
                x += __shfl_xor_sync(0xffffffffu, x, 8);
                x += __shfl_xor_sync(0xffffffffu, x, 16);
                if (lane < 4) column[quarter][8 * (k >> 1) + col + (k & 1)] = x;
            }
            sync_128(id);
            const int64_t part = (int64_t)g.slot * 64 + h1;
            const int own = heads - h1;            // heads of this half
            if (quarter == 0 && lane < 4)
#pragma unroll
                for (int k = 0; k < 2 * J; ++k) {
                    const int h = 8 * (k >> 1) + col + (k & 1);
                    const float x = (column[0][h] + column[1][h]) + (column[2][h] + column[3][h]);
                    factor[h] = g.slot < 0 ? 1.f / x : 1.f;
                    if (g.slot >= 0 && h < own) a.part_ml[part + h] = make_float2(m[k], x);
                }
            wait(&bars.pv_done, (uint32_t)(it - 1) & 1u);
            dead = any_of_128(id, dead);
            tc_fence_after();
#pragma unroll 1
            for (int mb = 0; mb < nm; ++mb) {
                const int dim = mb * 128 + 32 * quarter + lane;
                __nv_bfloat16* o = (__nv_bfloat16*)a.io.o + g.block * a.io.o_block_stride + h1 * a.io.o_head_stride + (dim & ~1);
                constexpr int W = NH < 16 ? NH : 16;
#pragma unroll
                for (int c = 0; c < NH; c += W) {
                    float v[W];
                    if constexpr (W == 16) tc_ld16(tmem + lanes + kColO + mb * N + h1 + c, v);
                    else tc_ld8(tmem + lanes + kColO + mb * N + h1 + c, v);
                    if (dead) continue;
                    if (g.slot >= 0) {
#pragma unroll
                        for (int e = 0; e < W; ++e)
                            if (c + e < own) a.part_o[(part + c + e) * L + dim] = v[e];
                    } else {
                        // two heads at a time: an even lane takes its own and its neighbour's element of the first, an odd one
                        // of the second
#pragma unroll
                        for (int e = 0; e < W; e += 2) {
                            const float x = mul_keep(v[e], factor[c + e]), y = mul_keep(v[e + 1], factor[c + e + 1]);
                            const float other = __shfl_xor_sync(0xffffffffu, (lane & 1) ? x : y, 1);
                            const uint32_t w = (lane & 1) ? bf_pack(other, y) : bf_pack(x, other);
                            const int h = c + e + (lane & 1);
                            if (h < own) *reinterpret_cast<uint32_t*>(o + h * a.io.o_head_stride) = w;
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&bars.o_empty));
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 13) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" :: "r"(tmem) : "memory");
    }
}

// ---------------------------------------------------------------- joining a cut block's parts
// (The last CTA of a block joining its parts itself was slower wherever blocks were cut, 83 us for 57 and 109 for 61: it reads
// alone what here the whole device reads.)
// One unit = 128 elements of a (cut block, head), four per lane of a warp.  Where no block has more than kFewParts parts a warp
// takes a unit by itself, else a CTA's eight warps share a unit's parts.  (Short code: it runs once or twice per launch, so
// fetching its instructions is part of its time.)
constexpr int kJoinWarps = 8, kFewParts = 8, kJoinBatch = 4, kJoinPerSm = 4;
// (the values keep what lies below the normal range; the sums are far above it)
__device__ __forceinline__ void scale_part(float4& v, float& l, float f) {
    v = make_float4(mul_keep(v.x, f), mul_keep(v.y, f), mul_keep(v.z, f), mul_keep(v.w, f));
    l *= f;
}
__device__ __forceinline__ void add_part(float4& v, float& l, const uint4& w, float wl, float f) {
    v.x = fma_keep(f, __uint_as_float(w.x), v.x);
    v.y = fma_keep(f, __uint_as_float(w.y), v.y);
    v.z = fma_keep(f, __uint_as_float(w.z), v.z);
    v.w = fma_keep(f, __uint_as_float(w.w), v.w);
    l = fmaf(f, wl, l);
}
__device__ __forceinline__ float2 ld_f2(const float2* p) {
    float2 v;
    asm volatile("ld.global.v2.f32 {%0,%1}, [%2];\n" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__global__ void __launch_bounds__(kJoinWarps * 32, kJoinPerSm) latent_join_kernel(const __grid_constant__ decode_args a) {
    __shared__ int list[3][kSms];             // block, parts, group
    __shared__ int count[kJoinWarps];
    __shared__ uint4 acc[kJoinWarps][32];
    __shared__ float2 sums[kJoinWarps];
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    static_assert(kSms <= kJoinWarps * 32, "a thread per group");
    int2 cut = make_int2(-1, 0);              // the cuts in their order, which all CTAs have to agree on
    if ((int)threadIdx.x < a.groups) cut = make_int2(ld_i32(&a.cuts[threadIdx.x].x), ld_i32(&a.cuts[threadIdx.x].y));
    const uint32_t has = __ballot_sync(0xffffffffu, cut.x >= 0);
    if (lane == 0) count[warp] = __popc(has);
    const bool shared = __syncthreads_or(cut.y > kFewParts);
    int n_list = 0, at = __popc(has & ((1u << lane) - 1));
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
        if (w < warp) at += count[w];
        n_list += count[w];
    }
    if (cut.x >= 0) {
        // (what the workspace says is not followed outside of it)
        if (cut.x >= a.B || cut.y < 1 || cut.y > a.groups - (int)threadIdx.x) {
            atomicCAS(a.t.header, 0, kStatusInvalid);
            cut = make_int2(0, 0);
        }
        list[0][at] = cut.x;
        list[1][at] = cut.y;
        list[2][at] = (int)threadIdx.x;
    }
    __syncthreads();
    const int quarters = a.L / 128, units = a.H * quarters;      // per cut block
    const int per = shared ? units : (units + kJoinWarps - 1) / kJoinWarps, n_work = n_list * per;
    for (int work = blockIdx.x; work < n_work; work += gridDim.x) {
        const int c = work / per, unit = shared ? work - c * per : (work - c * per) * kJoinWarps + warp;
        const int n = list[1][c], g0 = list[2][c];
        if (n < 1) continue;
        const bool on = unit < units;
        const int head = on ? unit / quarters : 0, e = (on ? unit % quarters : 0) * 128 + lane * 4;
        const int hg = head / a.group_heads;
        const int64_t step = 2 * (int64_t)a.head_groups * 64, row0 = ((int64_t)(2 * g0 + 1) * a.head_groups + hg) * 64 + head - hg * a.group_heads,
                      row1 = row0 - (int64_t)a.head_groups * 64;            // part 0; part k > 0 is at row1 + k * step
        // the parts of this warp, a batch in flight at a time, with a running reference
        const int k0 = shared ? warp : 0, dk = shared ? kJoinWarps : 1;
        float m = kLowest, l = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = k0; k < n; k += kJoinBatch * dk) {
            float2 ml[kJoinBatch];
            uint4 w[kJoinBatch];
#pragma unroll
            for (int i = 0; i < kJoinBatch; ++i) {
                const int at = k + i * dk;
                ml[i] = make_float2(kLowest, 0.f);
                w[i] = make_uint4(0, 0, 0, 0);
                if (at < n) {
                    const int64_t row = at == 0 ? row0 : row1 + at * step;
                    w[i] = ld_v4(a.part_o + row * a.L + e);
                    ml[i] = ld_f2(a.part_ml + row);
                }
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < kJoinBatch; ++i) top = fmaxf(top, ml[i].x);
            scale_part(v, l, exp2f(m - top));
            m = top;
#pragma unroll
            for (int i = 0; i < kJoinBatch; ++i) add_part(v, l, w[i], ml[i].y, exp2f(ml[i].x - m));
        }
        if (shared) {
            if (lane == 0) sums[warp] = make_float2(m, l);
            acc[warp][lane] = make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
            __syncthreads();
            if (warp == 0) {
                float top = m;
                for (int k = 1; k < kJoinWarps; ++k) top = fmaxf(top, sums[k].x);
                scale_part(v, l, exp2f(m - top));
                for (int k = 1; k < kJoinWarps; ++k) add_part(v, l, acc[k][lane], sums[k].y, exp2f(sums[k].x - top));
            }
        }
        if (on && (!shared || warp == 0)) {
            const float f = 1.f / l;
            *reinterpret_cast<uint2*>((__nv_bfloat16*)a.io.o + list[0][c] * a.io.o_block_stride + head * a.io.o_head_stride + e) =
                make_uint2(bf_pack(mul_keep(v.x, f), mul_keep(v.y, f)), bf_pack(mul_keep(v.z, f), mul_keep(v.w, f)));
        }
        if (shared) __syncthreads();
    }
}

// Queries [B, H, elements] as boxes of N heads: 64 elements x heads (x column blocks) x one block.
bool make_q_map(CUtensorMap* map, const void* q, int B, int H, int64_t block_stride, int64_t head_stride, int columns, int N) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t hs = (cuuint64_t)(H > 1 ? head_stride : 64 * columns) * 2, bs = (cuuint64_t)(B > 1 ? block_stride : 64 * columns) * 2;
    const cuuint64_t dims4[4] = {64, (cuuint64_t)H, (cuuint64_t)columns, (cuuint64_t)B}, strides4[3] = {hs, 128, bs};
    const cuuint32_t box4[4] = {64, (cuuint32_t)N, (cuuint32_t)columns, 1}, elem[4] = {1, 1, 1, 1};
    const cuuint64_t dims3[3] = {64, (cuuint64_t)H, (cuuint64_t)B}, strides3[2] = {hs, bs};
    const cuuint32_t box3[3] = {64, (cuuint32_t)N, 1};
    const bool four = columns > 1;
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, four ? 4 : 3, const_cast<void*>(q), four ? dims4 : dims3, four ? strides4 : strides3,
              four ? box4 : box3, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool io_ok(const cpa_latent_io* io, int B, int H, int L) {
    if (!io || !io->q_latent || !io->q_rope || !io->o || !latent_aligned(io->q_latent, 16) || !latent_aligned(io->q_rope, 16) ||
        !latent_aligned(io->o, 16))
        return false;
    // (strides of a single block or head are not looked at)
    for (int64_t s : {B > 1 ? io->q_latent_block_stride : 8, H > 1 ? io->q_latent_head_stride : 8, B > 1 ? io->q_rope_block_stride : 8,
                      H > 1 ? io->q_rope_head_stride : 8}) {
        // queries are read through tensor maps: whole pieces, and positive below 2^40 bytes
        if (s % 8 != 0 || s <= 0 || s >= (int64_t)1 << 39) return false;
    }
    if ((B > 1 && io->o_block_stride % 8 != 0) || (H > 1 && io->o_head_stride % 8 != 0)) return false;
    if (io->o == io->q_latent || io->o == io->q_rope) return false;
    // heads of the output must not share elements: blocks of heads, or heads of blocks
    const int64_t bs = B > 1 ? io->o_block_stride : INT64_MAX, hs = H > 1 ? io->o_head_stride : INT64_MAX;
    if (bs < L || hs < L) return false;
    return B == 1 || H == 1 || bs >= (H - 1) * hs + L || hs >= (B - 1) * bs + L;
}

// The pool as page-wise boxes: 64 elements x 8 tokens x column blocks x 2 groups of 8 tokens, which lands as
// [group of 8 tokens][column block][8 rows of 128 bytes, swizzled]: uniform strides in tokens and in elements for both products.
bool make_page_map(CUtensorMap* map, const void* pool, int64_t pages, int L, int columns) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t row = (cuuint64_t)(L + kRopeDim) * 2, nc = (cuuint64_t)L / 64 + 1;
    const cuuint64_t dims[4] = {64, 8, nc, (cuuint64_t)pages * 2};
    const cuuint64_t strides[3] = {row, 128, row * 8};
    const cuuint32_t box[4] = {64, 8, (cuuint32_t)columns, 2};
    const cuuint32_t elem[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, box, elem,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct decode_shape { int groups, head_groups, group_heads, n; };
decode_shape shape_of(const cpa_latent_config& c) {
    decode_shape s;
    s.head_groups = c.num_heads > 64 ? 2 : 1;
    s.group_heads = (c.num_heads + s.head_groups - 1) / s.head_groups;
    s.n = s.group_heads <= 16 ? 16 : s.group_heads <= 32 ? 32 : 64;
    const int sms = c.num_sms ? std::min(c.num_sms, kSms) : kSms;
    s.groups = std::max(1, sms / s.head_groups);
    return s;
}
struct workspace { int64_t ml, o, cuts, bytes; };
workspace workspace_of(const cpa_latent_config& c) {
    const decode_shape s = shape_of(c);
    const int64_t rows = (int64_t)s.groups * 2 * s.head_groups * 64;
    workspace w = {};
    w.ml = 0;
    w.o = rows * 8;
    w.cuts = w.o + rows * c.latent_dim * 4;
    w.bytes = (w.cuts + s.groups * 8 + 255) / 256 * 256 + 256;       // and what its alignment may take
    return w;
}

template <int L, int N>
int launch(const CUtensorMap (&map)[4], const decode_args& a, cudaStream_t st) {
    static std::atomic<bool> configured_dev[64];
    int dev_id = 0;
    if (cudaGetDevice(&dev_id) != cudaSuccess || dev_id < 0 || dev_id >= 64) {
        (void)cudaGetLastError();
        return CPA_ECUDA;
    }
    constexpr int smem = DecodeShape<L, N>::kSmem;
    if (!configured_dev[dev_id].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(latent_decode_kernel<L, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
            (void)cudaGetLastError();
            return CPA_ECUDA;
        }
        configured_dev[dev_id].store(true, std::memory_order_relaxed);
    }
    return q8_launch_smem(latent_decode_kernel<L, N>, a.groups, kDecodeThreads, smem, st, map[0], map[1], map[2], a);
}
template <int N>
int launch_latent(const CUtensorMap (&map)[4], const decode_args& a, cudaStream_t st) {
    switch (a.L) {
        case 128: return launch<128, N>(map, a, st);
        case 256: return launch<256, N>(map, a, st);
        case 384: return launch<384, N>(map, a, st);
        default: return launch<512, N>(map, a, st);
    }
}

int decode(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables, const cpa_rope_config* rope,
           const uint64_t* d_turns, const cpa_latent_io* io, const void* x, int64_t x_row, const void* weight, const int32_t* d_first,
           const int32_t* d_lens, int32_t* d_lens_out, const int32_t* d_active, const void* pool, void* d_workspace, void* stream) {
    const decode_shape s = shape_of(*cfg);
    const workspace w = workspace_of(*cfg);
    decode_args a = {};
    a.t = q8_view(latent_tables_cfg(*cfg), *dims, d_tables);
    a.io = *io;
    a.turns = d_turns;
    a.first = d_first;
    a.lens = d_lens;
    a.active = d_active;
    a.x = (const __nv_bfloat16*)x;
    a.weight = (const __nv_bfloat16*)weight;
    a.x_row = x_row;
    a.lens_out = d_lens_out;
    a.pool = (__nv_bfloat16*)const_cast<void*>(pool);
    char* ws = (char*)(((uintptr_t)d_workspace + 255) & ~(uintptr_t)255);      // (the pair kernel stores 32 bytes at a time)
    a.part_ml = (float2*)(ws + w.ml);
    a.part_o = (float*)(ws + w.o);
    a.cuts = (int2*)(ws + w.cuts);
    a.B = dims->num_blocks;
    a.H = cfg->num_heads;
    a.L = cfg->latent_dim;
    a.groups = s.groups;
    a.head_groups = s.head_groups;
    a.group_heads = s.group_heads;
    a.interleaved = rope && rope->layout == CPA_ROPE_INTERLEAVED;
    a.scale_log2 = cfg->scale * 1.4426950408889634f;
    a.amplitude = rope ? (float)rope->amplitude : 1.f;
    a.eps = cfg->norm_eps;
    a.list_words = dims->page_capacity;
    CUtensorMap map[4];
    if (!make_page_map(&map[0], pool, dims->num_pages, a.L, a.L / 64 + 1) ||
        (s.head_groups == 2 && !make_page_map(&map[3], pool, dims->num_pages, a.L, a.L / 128)) ||
        !make_q_map(&map[1], io->q_latent, a.B, a.H, io->q_latent_block_stride, io->q_latent_head_stride, a.L / 64, s.n) ||
        !make_q_map(&map[2], io->q_rope, a.B, a.H, io->q_rope_block_stride, io->q_rope_head_stride, 1, s.n))
        return CPA_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    const int rc = s.head_groups == 2 ? latent_decode_pairs(map, &a, stream)
                   : s.n == 16        ? launch_latent<16>(map, a, st)
                   : s.n == 32        ? launch_latent<32>(map, a, st)
                                      : launch_latent<64>(map, a, st);
    if (rc != CPA_OK) return rc;
    return q8_launch(latent_join_kernel, kJoinPerSm * kSms, kJoinWarps * 32, st, a);
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
    return rc != CPA_OK ? rc : workspace_of(*cfg).bytes;
}

extern "C" int cpa_latent_decode(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                                 const cpa_latent_io* io, const int32_t* d_lens, const int32_t* d_active, const void* pool,
                                 void* d_workspace, void* stream) {
    const int rc = check(cfg, dims, d_tables, io, d_lens, d_active, pool, d_workspace);
    if (rc != CPA_OK) return rc;
    return decode(cfg, dims, d_tables, nullptr, nullptr, io, nullptr, 0, nullptr, nullptr, d_lens, nullptr, d_active, pool, d_workspace,
                  stream);
}

extern "C" int cpa_latent_step(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                               const cpa_rope_config* rope, const uint64_t* d_turns, const cpa_latent_io* io, const void* x,
                               int64_t x_row_stride, const void* norm_weight, const int32_t* d_first, const int32_t* d_lens,
                               int32_t* d_lens_out, const int32_t* d_active, void* pool, void* d_workspace, void* stream) {
    int rc = check(cfg, dims, d_tables, io, d_lens, d_active, pool, d_workspace);
    if (rc != CPA_OK) return rc;
    if (!x || !d_lens_out || d_lens_out == d_lens || !latent_aligned(x, 2) || !latent_aligned(norm_weight, 16) ||
        !latent_aligned(d_turns, 8) || !latent_aligned(d_first, 4) || !latent_aligned(d_lens_out, 4) ||
        (d_turns != nullptr) != (rope != nullptr) || (rope && (!rope_config_ok(rope) || rope->rope_dim != kRopeDim)) ||
        (dims->num_blocks > 1 && x_row_stride < cfg->latent_dim + kRopeDim))
        return CPA_EINVAL;
    return decode(cfg, dims, d_tables, rope, d_turns, io, x, x_row_stride, norm_weight, d_first, d_lens, d_lens_out, d_active, pool,
                  d_workspace, stream);
}
