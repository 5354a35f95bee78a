// Expanded latent attention: varlen causal prefill with keys of 128 + 64 elements, whose positional part is shared by the heads,
// and values of 128, on the 5th-generation tensor cores.
//
//     S = Q K^T,  K = [k_nope | r]       12 MMAs of 16 elements per 128 x 128 scores: eight over the head's key part, four over r
//     P = exp2(scale S - m),  O += P V   as in the other prefill: P over S in tensor memory, O in tensor memory, online softmax in
//                                        fp32 registers, one thread per query row
//
// The unit of work is the plan's (block, q item, head): 256 query rows as two 128-row sub-tiles that share every K/V tile, with a
// softmax warpgroup each; the grid is persistent and walks the plan's schedule.  The keys are never put together in memory: a
// tile's three column blocks come from where they lie, two from the head's part of kv and one from the rows of r.
//
// Shared memory: the queries take 96 KB, which leaves 128 KB.  K and V tiles of 128 keys (48 and 32 KB) therefore go through
// one ring of eight 16 KB pieces in the order of their use: a K tile is three pieces (column blocks of 128 keys x 64 elements), a
// V tile two (64 keys x 128 elements).  While a V tile and the next K tile are in use three pieces are under way; rings of their
// own would hold two K tiles and one V tile, with nothing under way while the one V tile is read.
// A lone sub-tile (a block's last 128 rows, or all of a short block) takes the two sub-tiles' places in turn, and the two score
// buffers step by step: the next unit's queries are there and its first scores are made while this one's last softmax and
// output run.  A last tile of at most 64 keys is worked through in groups of 32, by the warps that have rows of the block and with
// the MMAs that its keys need.  (177 blocks of 18 tokens, 20 heads: 82 us without either, 72 with the first, 42 with both.  Working every
// last tile through in groups spares half of a diagonal's exponentials and was slower, 3.4 ms for the long prompts below: the
// loop of whole tiles loses registers to it.  Loading only the parts of a short tile that hold rows: 63 us for 42.)
// Tensor memory: two score buffers of 128 columns (one per sub-tile, or step by step for lone ones) and two outputs of 128.
// Warps 0-3, 4-7 softmax + epilogue of sub-tile 0, 1; warp 8 TMA producer; warp 9 MMA issuer and owner of the tensor memory;
// warps 10-11 idle, they complete the warpgroup whose registers go to the softmax.
// Keys behind a block's end are the next block's: their scores are masked by index and those of their V rows that an MMA reads
// are cleared, so that what they hold (infinities, NaN) stays theirs.
// Measured: 32 prompts of 1024..8192 tokens, 16 heads: 3.33 ms, 1.05 PFLOP/s of the products below the diagonal, in a row (3.20 to 3.35,
// under the power limit; a single call 2.96 ms).  A pair of steps (both sub-tiles, one K/V tile) takes 3380 cycles, of which the
// tensor core is busy 2560; the rest is the softmax of a sub-tile waiting for its scores: buffers for the scores of the next tile as
// well would fit with the weights in place of the oldest scores only, and were slower (3.48 ms: both softmaxes then run at once and
// slow one another down).  9 odd blocks of 1..700 tokens, 16 heads: 24-25 us, the work of all items with their fixed part (the longest
// block, 592 tokens, alone 14.4; the other eight 24.3).
// Every mbarrier wait is bounded (see prefill_tc.cu).
#include <atomic>

#include "cpa_tcgen05.cuh"
#include "latent.cuh"

namespace {

constexpr int kPieces = 8;                                    // of the ring
constexpr uint32_t kPieceBytes = 16384;
constexpr int kTilePieces = 5;                                // K: 3, V: 2
constexpr int kShortKeys = 64;                                // a last tile of at most so many keys is worked through in parts
constexpr uint32_t kQTileBytes = 3 * kPieceBytes;             // 128 rows x 192 elements
constexpr int kV = 128;                                       // elements of a value
constexpr uint32_t kOutCol = 256;                             // outputs behind the two score buffers

struct __align__(8) PrefillBarriers {
    uint64_t q_full[2], q_empty[2], full[kPieces], empty[kPieces];
    uint64_t s_full[2][4], p_half[2][4], p_full[2][4];   // [sub-tile][its step mod 4]
    uint64_t pv_done[2];              // a sub-tile's step is in its output
    uint64_t drain;
    uint32_t tmem_base;
};
constexpr int kPrefillSmem = 2 * (int)kQTileBytes + kPieces * (int)kPieceBytes + (int)sizeof(PrefillBarriers);

// See TcWork in prefill_tc.cu: sub-tile u sees KV tiles 0 .. t0 + u, the last of which touches the diagonal.
struct PrefillWork { int h, tok0, L, q0, t0, n_sub, n_total; bool valid; };

// A count for each sub-tile, in registers where the sub-tile is known at run time only.
struct pair_count {
    uint32_t n0 = 0, n1 = 0;
    __device__ __forceinline__ uint32_t of(int u) const { return u ? n1 : n0; }
    __device__ __forceinline__ void add(int u) {
        n0 += u ? 0u : 1u;
        n1 += u ? 1u : 0u;
    }
};
// by one thread; descriptors as halves
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %5, 0;\n mov.b64 da, {%1, %3};\n mov.b64 db, {%2, %3};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n}\n"
        :: "r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 db;\n setp.ne.b32 p, %5, 0;\n mov.b64 db, {%2, %3};\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}\n"
        :: "r"(d), "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" :: "r"(bar) : "memory");
}

__global__ void __launch_bounds__(kThreads, 1)
latent_prefill_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                      const __grid_constant__ CUtensorMap tm_r, const __grid_constant__ CUtensorMap tm_v, __nv_bfloat16* o,
                      cpa_dev_index ix, int H, int q_rows, float scale_log2, int n_rounds) {
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem), s_q = base, s_ring = base + 2 * kQTileBytes;
    PrefillBarriers& bars = *reinterpret_cast<PrefillBarriers*>(smem + 2 * kQTileBytes + kPieces * kPieceBytes);
    if (base & 1023u) {              // swizzled tiles would be misread
        if (threadIdx.x == 0) atomicCAS(ix.status, 0, kStatusInvalid);
        return;
    }
    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
    const int G = gridDim.x;
    // unit of round k, with the next rounds' schedule entry and item record in flight
    auto fetch_code = [&](int k) { return k < n_rounds ? __ldg(ix.prefill_sched + (int64_t)k * G + blockIdx.x) : -1; };
    struct Rec { int4 a; int h; };
    auto fetch = [&](int code, Rec& r) {
        r.a = make_int4(0, 0, 0, 0);
        r.h = 0;
        if (code >= 0) {
            const int item = code / H;
            r.h = code - item * H;
            r.a = __ldg(reinterpret_cast<const int4*>(ix.prefill_items) + item);
        }
    };
    auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    auto decode = [&](const Rec& r, PrefillWork& w) {
        w.valid = r.a.y > 0;
        w.h = r.h;
        w.tok0 = r.a.x;
        w.L = r.a.y;
        w.q0 = (r.a.z & 0xFFFF) * q_rows;
        w.t0 = w.q0 / kTileM;
        w.n_sub = (q_rows > kTileM && w.L - w.q0 > kTileM) ? 2 : 1;
        w.n_total = w.t0 + w.n_sub;
    };
    auto bar = [](uint64_t* p) { return smem_u32(p); };

    if (threadIdx.x == 0) {
        for (int u = 0; u < 2; ++u) {
            mbar_init(bar(&bars.q_full[u]), 1);
            mbar_init(bar(&bars.q_empty[u]), 1);
            mbar_init(bar(&bars.pv_done[u]), 1);
            for (int i = 0; i < 4; ++i) {
                mbar_init(bar(&bars.s_full[u][i]), 1);
                mbar_init(bar(&bars.p_half[u][i]), 128);
                mbar_init(bar(&bars.p_full[u][i]), 128);
            }
        }
        for (int i = 0; i < kPieces; ++i) {
            mbar_init(bar(&bars.full[i]), 1);
            mbar_init(bar(&bars.empty[i]), 1);
        }
        mbar_init(bar(&bars.drain), 1);
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" :: "r"(smem_u32(&bars.tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem_base;
    bool dead = false;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" :: "n"(kRegsControl));
        if (warp == 8 && elect_one()) {
            // ------------------------------------------------------------ TMA producer
            int n = 0;                    // pieces loaded: slot n % kPieces, use n / kPieces
            pair_count q_loads;
            int lone = 0;
            PrefillWork w;
            Rec rec;
            fetch(fetch_code(0), rec);
            int code = fetch_code(1);
            for (int k = 0; k < n_rounds && !dead; ++k) {
                decode(rec, w);
                fetch(code, rec);
                code = fetch_code(k + 2);
                if (!w.valid) continue;
                auto load_q = [&](int u, int row) {
                    tc_wait(bar(&bars.q_empty[u]), (q_loads.of(u) & 1u) ^ 1u, dead, ix.status);
                    if (dead) return;
                    q_loads.add(u);
                    mbar_expect_tx(bar(&bars.q_full[u]), kQTileBytes);
#pragma unroll
                    for (int c = 0; c < 3; ++c)
                        tma_load_2d(s_q + u * kQTileBytes + c * kPieceBytes, &tm_q, w.h * 192 + 64 * c, w.tok0 + row,
                                    bar(&bars.q_full[u]));
                };
                // slot of the next piece, once it is free; its barrier expects the whole piece
                auto next = [&]() {
                    const int s = n % kPieces;
                    tc_wait(bar(&bars.empty[s]), ((uint32_t)(n / kPieces) & 1u) ^ 1u, dead, ix.status);
                    if (!dead) {
                        mbar_expect_tx(bar(&bars.full[s]), kPieceBytes);
                        ++n;
                    }
                    return s;
                };
                if (w.n_sub == 2) {
                    load_q(0, w.q0);
                    load_q(1, w.q0 + kTileM);
                } else {
                    load_q(lone++ & 1, w.q0);
                }
                for (int j = 0; j < w.n_total && !dead; ++j) {
                    const int row = w.tok0 + j * kTileN;
#pragma unroll
                    for (int c = 0; c < 3; ++c) {
                        const int s = next();
                        if (dead) break;
                        if (c < 2) tma_load_2d(s_ring + s * kPieceBytes, &tm_k, w.h * 256 + 64 * c, row, bar(&bars.full[s]));
                        else tma_load_2d(s_ring + s * kPieceBytes, &tm_r, 0, row, bar(&bars.full[s]));
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (dead) break;
                        const int s = next();
                        if (dead) break;
                        tma_load_2d(s_ring + s * kPieceBytes, &tm_v, w.h * 256 + 128, row + 64 * c, bar(&bars.full[s]));
                        tma_load_2d(s_ring + s * kPieceBytes + kPieceBytes / 2, &tm_v, w.h * 256 + 192, row + 64 * c, bar(&bars.full[s]));
                    }
                }
            }
            if (dead) {      // copies issued last may still be on their way into this CTA's shared memory
                for (int u = 0; u < 2; ++u)
                    if (q_loads.of(u) > 0) mbar_drain(bar(&bars.q_full[u]), (q_loads.of(u) - 1u) & 1u, kDrainLimit);
                for (int t = max(0, n - kPieces); t < n; ++t)
                    mbar_drain(bar(&bars.full[t % kPieces]), (uint32_t)(t / kPieces) & 1u, kDrainLimit);
            }
        } else if (warp == 9 && elect_one()) {
            // ------------------------------------------------------------ MMA issuer
            constexpr uint32_t idesc_qk = instr_desc(kTileM, kTileN, false), idesc_pv = instr_desc(kTileM, kV, true);
            const uint64_t dk = smem_desc(0, 16, 1024), dv = smem_desc(0, kPieceBytes / 2, 1024);
            const uint32_t k_hi = (uint32_t)(dk >> 32), v_hi = (uint32_t)(dv >> 32);
            const uint32_t q_lo = (uint32_t)dk | (s_q >> 4), k_lo = (uint32_t)dk | (s_ring >> 4), v_lo = (uint32_t)dv | (s_ring >> 4);
            pair_count n_qk, n_pv, q_uses;
            int kt0 = 0;                                    // K/V tiles of earlier units
            // piece c of tile kt: 0-2 of K, 3-4 of V
            auto slot = [](int kt, int c) { return (uint32_t)(kt * kTilePieces + c) % kPieces; };
            auto wait_piece = [&](int kt, int c) {
                const uint32_t i = (uint32_t)(kt * kTilePieces + c);
                tc_wait(bar(&bars.full[i % kPieces]), (i / kPieces) & 1u, dead, ix.status);
            };
            auto release = [&](int kt, int c0, int c1) {
                for (int c = c0; c < c1; ++c) commit(bar(&bars.empty[slot(kt, c)]));
            };
            auto qk = [&](int u, int buf, int kt) {         // S[buf] = Q_u K[tile kt]^T
                const uint32_t a = q_lo + u * (kQTileBytes >> 4), d = tmem + buf * 128;
#pragma unroll
                for (int c = 0; c < 3; ++c) {
                    wait_piece(kt, c);
                    if (dead) return;
                    tc_fence_after();
                    const uint32_t b = k_lo + slot(kt, c) * (kPieceBytes >> 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_ss(d, a + c * (kPieceBytes >> 4) + k * 2, b + k * 2, k_hi, idesc_qk, (c | k) != 0);
                }
                commit(bar(&bars.s_full[u][n_qk.of(u) & 3u]));
                n_qk.add(u);
            };
            // O_u += P[buf] V[tile kt], 64 keys at a time, `ks` times 16 keys in all
            auto pv = [&](int u, int buf, int kt, uint32_t acc0, int ks) {
                const uint32_t d = tmem + kOutCol + u * kV, a = tmem + buf * 128, n = n_pv.of(u);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    wait_piece(kt, 3 + half);
                    tc_wait(bar(half ? &bars.p_full[u][n & 3u] : &bars.p_half[u][n & 3u]), (n >> 2) & 1u, dead, ix.status);
                    if (dead) return;
                    tc_fence_after();
                    const uint32_t b = v_lo + slot(kt, 3 + half) * (kPieceBytes >> 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (half * 4 + k < ks) mma_ts(d, a + half * 32 + k * 8, b + k * (2048 >> 4), v_hi, idesc_pv, half + k > 0 ? 1u : acc0);
                }
                commit(bar(&bars.pv_done[u]));
                n_pv.add(u);
            };
            auto steps_of = [](int keys) { return keys <= kShortKeys ? (keys + 15) / 16 : kTileN / 16; };
            auto wait_q = [&](int u) {
                tc_wait(bar(&bars.q_full[u]), q_uses.of(u) & 1u, dead, ix.status);
                q_uses.add(u);
            };
            // A lone sub-tile's output product waits until the scores of the step behind it are queued, the next unit's first one too.
            struct { int u, buf, kt, acc0, ks; bool on; } last = {0, 0, 0, 0, 0, false};
            auto finish = [&]() {
                if (!last.on || dead) return;
                pv(last.u, last.buf, last.kt, (uint32_t)last.acc0, last.ks);
                release(last.kt, 3, 5);
                last.on = false;
            };
            int lone = 0, lone_steps = 0;
            PrefillWork w;
            Rec rec;
            fetch(fetch_code(0), rec);
            int code = fetch_code(1);
            for (int rd = 0; rd < n_rounds && !dead; ++rd) {
                decode(rec, w);
                fetch(code, rec);
                code = fetch_code(rd + 2);
                if (!w.valid) continue;
                const int t0 = w.t0;
                if (w.n_sub == 2) {
                    finish();
                    wait_q(0);
                    // PV of a sub-tile's step, then the scores of its next one into the buffer that PV has read; the other
                    // sub-tile's softmax runs meanwhile
                    wait_q(1);
                    qk(0, 0, kt0);
                    qk(1, 1, kt0);
                    release(kt0, 0, 3);
                    if (t0 == 0) commit(bar(&bars.q_empty[0]));
                    for (int j = 0; j <= t0 && !dead; ++j) {      // tiles both sub-tiles have; sub-tile 1 also has tile t0 + 1
                        const int kt = kt0 + j;
                        pv(0, 0, kt, j > 0, 8);
                        if (j < t0) qk(0, 0, kt + 1);
                        if (j == t0 - 1) commit(bar(&bars.q_empty[0]));
                        pv(1, 1, kt, j > 0, 8);
                        release(kt, 3, 5);
                        qk(1, 1, kt + 1);
                        release(kt + 1, 0, 3);
                        if (j == t0) commit(bar(&bars.q_empty[1]));
                    }
                    if (!dead) pv(1, 1, kt0 + t0 + 1, 1u, steps_of(w.L - (t0 + 1) * kTileN));
                    release(kt0 + t0 + 1, 3, 5);
                } else {
                    const int u = lone++ & 1;
                    wait_q(u);
                    for (int j = 0; j <= t0 && !dead; ++j) {
                        const int buf = lone_steps++ & 1;
                        qk(u, buf, kt0 + j);
                        release(kt0 + j, 0, 3);
                        if (j == t0) commit(bar(&bars.q_empty[u]));
                        finish();
                        last = {u, buf, kt0 + j, j > 0, j == t0 ? steps_of(w.L - t0 * kTileN) : 8, true};
                    }
                }
                kt0 += w.n_total;
            }
            finish();
            if (dead) {      // MMAs queued before may still be running; tensor memory is not freed under them
                commit(bar(&bars.drain));
                mbar_drain(bar(&bars.drain), 0u, kDrainLimit);
            }
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" :: "n"(kRegsSoftmax));
        // ------------------------------------------------------------ softmax + epilogue (one warpgroup per sub-tile)
        const int u = warp >> 2, r = threadIdx.x & 127;                   // sub-tile; query row in it = TMEM lane
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_o = tmem + lane_addr + kOutCol + u * kV;
        uint32_t n_steps = 0;
        int kt0 = 0, lone = 0, lone_steps = 0;
        PrefillWork w;
        Rec rec;
        fetch(fetch_code(0), rec);
        int code = fetch_code(1);
        for (int rd = 0; rd < n_rounds; ++rd) {
            rec.a.x = uniform(rec.a.x); rec.a.y = uniform(rec.a.y); rec.a.z = uniform(rec.a.z); rec.h = uniform(rec.h);
            decode(rec, w);
            fetch(code, rec);
            code = uniform(fetch_code(rd + 2));
            if (!w.valid) continue;
            if (w.n_sub == 2 || u == (lone & 1)) {
                const int sub = w.n_sub == 2 ? u : 0;
                const int n_kv = w.t0 + 1 + sub;
                const int left = w.L - (n_kv - 1) * kTileN;                // keys of the last tile that are the block's
                const int n_full = left <= kShortKeys ? n_kv - 1 : n_kv;   // tiles that are worked through whole
                float m_used = -INFINITY, l_run = 0.f;
                for (int j = 0; j < n_full; ++j, ++n_steps) {
                    const uint32_t t_s = tmem + lane_addr + (w.n_sub == 2 ? u : (lone_steps + j) & 1) * 128;
                    tc_wait(bar(&bars.s_full[u][n_steps & 3u]), (n_steps >> 2) & 1u, dead, ix.status);
                    tc_fence_after();
                    uint32_t sv[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tc_ld32_nowait(t_s + c * 32, sv[c]);
                    tc_wait_ld();
                    if (j == n_kv - 1) {
                        // the diagonal: keys in the row's future become -inf, keys behind the block's end lose their V rows
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c * 32 + i > r) sv[c][i] = 0xff800000u;
                        if (left < kTileN) {      // (more than kShortKeys, so only rows of the second piece)
                            static_assert(kShortKeys == 64, "a last tile that is worked through whole reaches into its second V piece");
                            const uint32_t i = (uint32_t)((kt0 + j) * kTilePieces + 4);
                            tc_wait(bar(&bars.full[i % kPieces]), (i / kPieces) & 1u, dead, ix.status);
                            const int first = left - 64;
                            if (!dead)
                                for (int e = r; e < (64 - first) * 16; e += 128)
                                    *reinterpret_cast<uint4*>(smem + (s_ring - base) + (i % kPieces) * kPieceBytes + (e & 8) * (kPieceBytes / 16) +
                                                              (first + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
                            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                        }
                    }
                    float mxa[8];
#pragma unroll
                    for (int a = 0; a < 8; ++a)
                        mxa[a] = fmaxf(max3(__uint_as_float(sv[0][a]), __uint_as_float(sv[0][a + 8]), __uint_as_float(sv[0][a + 16])),
                                       __uint_as_float(sv[0][a + 24]));
#pragma unroll
                    for (int c = 1; c < 4; ++c)
#pragma unroll
                        for (int a = 0; a < 8; ++a) {
                            mxa[a] = max3(mxa[a], __uint_as_float(sv[c][a]), __uint_as_float(sv[c][a + 8]));
                            mxa[a] = max3(mxa[a], __uint_as_float(sv[c][a + 16]), __uint_as_float(sv[c][a + 24]));
                        }
                    const float mx = scale_log2 * max3(max3(mxa[0], mxa[1], mxa[2]), max3(mxa[3], mxa[4], mxa[5]), fmaxf(mxa[6], mxa[7]));
                    // the reference stays until the maximum is 2^8 above it (cancels in the division)
                    float alpha = 1.f;
                    if (mx > m_used + 8.f) {
                        alpha = m_used == -INFINITY ? 0.f : exp2f(m_used - mx);
                        m_used = mx;
                    }
                    if (j > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
                        tc_wait(bar(&bars.pv_done[u]), (n_steps - 1) & 1u, dead, ix.status);      // O_u holds every earlier tile
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < kV / 8; ++c) {
                            float v[8];
                            tc_ld8(t_o + c * 8, v);
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = mul_keep(v[e], alpha);
                            tc_st8(t_o + c * 8, v);
                        }
                    }
                    l_run *= alpha;
                    // weights in bf16, two keys per 32-bit column over the first 64 columns of S; the sum is of the rounded ones
                    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                    const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t pk[16];
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            float x0 = __uint_as_float(sv[c][i]), x1 = __uint_as_float(sv[c][i + 1]);
                            fma_x2(x0, x1, scale_log2, neg_m);
                            const uint32_t w2 = pack_bf16(exp2f(x0), exp2f(x1));
                            pk[i >> 1] = w2;
                            add_bf16x2(sum[(i >> 1) & 7], w2);
                        }
                        tc_st16(t_s + c * 16, pk);
                        if (c == 1) {      // the first 64 keys' MMAs may start
                            tc_wait_st();
                            tc_fence_before();
                            mbar_arrive(bar(&bars.p_half[u][n_steps & 3u]));
                        }
                    }
                    l_run += ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
                    tc_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(&bars.p_full[u][n_steps & 3u]));
                }
                if (n_full < n_kv) {
                    // ---- a last tile of few keys, and as many rows: 32 keys at a time, and only by the warps that have rows of the block (what the
                    // others' rows come to is not stored)
                    const int own = warp & 3, lane = r & 31, groups = (left + 31) / 32;
                    const uint32_t t_s = tmem + lane_addr + (w.n_sub == 2 ? u : (lone_steps + n_full) & 1) * 128;
                    tc_wait(bar(&bars.s_full[u][n_steps & 3u]), (n_steps >> 2) & 1u, dead, ix.status);
                    tc_fence_after();
                    if (left % 16 != 0) {      // the value rows behind the block's end that the MMA of the last 16 keys reads
                        const uint32_t i = (uint32_t)((kt0 + n_full) * kTilePieces + 3);
                        tc_wait(bar(&bars.full[i % kPieces]), (i / kPieces) & 1u, dead, ix.status);
                        if (!dead)
                            for (int e = r; e < (16 - left % 16) * 16; e += 128)
                                *reinterpret_cast<uint4*>(smem + (s_ring - base) + (i % kPieces) * kPieceBytes + (e & 8) * (kPieceBytes / 16) +
                                                          (left + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
                        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    }
                    if (own < groups) {
                        float mx = -INFINITY;
#pragma unroll 1
                        for (int c = 0; c <= own; ++c) {
                            float v[32];
                            tc_ld32(t_s + c * 32, v);
#pragma unroll
                            for (int i = 0; i < 32; ++i) mx = fmaxf(mx, c == own && i > lane ? -INFINITY : v[i]);
                        }
                        mx *= scale_log2;
                        float alpha = 1.f;
                        if (mx > m_used + 8.f) {
                            alpha = m_used == -INFINITY ? 0.f : exp2f(m_used - mx);
                            m_used = mx;
                        }
                        if (n_full > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
                            tc_wait(bar(&bars.pv_done[u]), (n_steps - 1) & 1u, dead, ix.status);
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < kV / 8; ++c) {
                                float v[8];
                                tc_ld8(t_o + c * 8, v);
#pragma unroll
                                for (int e = 0; e < 8; ++e) v[e] = mul_keep(v[e], alpha);
                                tc_st8(t_o + c * 8, v);
                            }
                        }
                        l_run *= alpha;
                        const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
#pragma unroll 1
                        for (int c = 0; c < groups; ++c) {
                            uint32_t pk[16];
                            if (c <= own) {
                                float v[32];
                                tc_ld32(t_s + c * 32, v);
#pragma unroll
                                for (int i = 0; i < 32; i += 2) {
                                    float x0 = c == own && i > lane ? -INFINITY : v[i], x1 = c == own && i + 1 > lane ? -INFINITY : v[i + 1];
                                    fma_x2(x0, x1, scale_log2, neg_m);
                                    pk[i >> 1] = pack_bf16(exp2f(x0), exp2f(x1));
                                    add_bf16x2(l_run, pk[i >> 1]);
                                }
                            } else {
#pragma unroll
                                for (int i = 0; i < 16; ++i) pk[i] = 0;
                            }
                            tc_st16(t_s + c * 16, pk);
                        }
                        tc_wait_st();
                    }
                    tc_fence_before();
                    mbar_arrive(bar(&bars.p_half[u][n_steps & 3u]));
                    mbar_arrive(bar(&bars.p_full[u][n_steps & 3u]));
                    ++n_steps;
                }
                // ---- epilogue: O / l; thread r owns row r.  O_u is overwritten by the next unit's first PV, which waits for
                // this warpgroup's next weights.
                tc_wait(bar(&bars.pv_done[u]), (n_steps - 1) & 1u, dead, ix.status);
                tc_fence_after();
                const float inv = 1.f / l_run;
                auto two = [&](float x, float y) { return pack_bf16(mul_keep(x, inv), mul_keep(y, inv)); };      // (outputs below the normal range too)
                const bool row_ok = !dead && r < w.L - (w.q0 + sub * kTileM);     // rows behind the block's end are not stored
                __nv_bfloat16* dst = o + ((int64_t)(w.tok0 + w.q0 + sub * kTileM + r) * H + w.h) * kV;
#pragma unroll
                for (int c = 0; c < kV / 32; ++c) {
                    float v[32];
                    tc_ld32(t_o + c * 32, v);
                    if (row_ok) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)
                            *reinterpret_cast<uint4*>(dst + c * 32 + i) =
                                make_uint4(two(v[i], v[i + 1]), two(v[i + 2], v[i + 3]), two(v[i + 4], v[i + 5]), two(v[i + 6], v[i + 7]));
                    }
                }
                tc_fence_before();
            }
            if (w.n_sub == 1) {
                ++lone;
                lone_steps += w.n_total;
            }
            kt0 += w.n_total;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" :: "r"(tmem) : "memory");
    }
}

// 2-D view [rows][cols] of rows `stride` elements apart; box = 64 cols x `box_rows`.
bool make_rows_map(CUtensorMap* map, const void* ptr, int64_t rows, int64_t cols, int64_t stride, int box_rows) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    const cuuint32_t elem[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box, elem,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
    out->q_tile_rows = CPA_Q_TILE_LATENT;
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
    // the attribute is per device: remember which devices have it (relaxed flags: setting it twice is harmless)
    static std::atomic<bool> configured_dev[64];
    int dev_id = 0;
    if (cudaGetDevice(&dev_id) != cudaSuccess || dev_id < 0 || dev_id >= 64) {
        (void)cudaGetLastError();
        return CPA_ECUDA;
    }
    if (!configured_dev[dev_id].load(std::memory_order_relaxed)) {
        cudaFuncAttributes attr;
        if (cudaFuncGetAttributes(&attr, latent_prefill_kernel) != cudaSuccess ||
            cudaFuncSetAttribute(latent_prefill_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPrefillSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return CPA_ECUDA;
        }
        // the register split in the kernel may only hand out what the launch allocates
        if (attr.numRegs * kThreads < 2 * 128 * kRegsSoftmax + 128 * kRegsControl) return CPA_EUNSUPPORTED;
        configured_dev[dev_id].store(true, std::memory_order_relaxed);
    }
    const int64_t T = plan->total_tokens, H = cfg->num_heads;
    CUtensorMap tm_q, tm_k, tm_r, tm_v;
    if (!make_rows_map(&tm_q, q, T, H * 192, H * 192, 128) || !make_rows_map(&tm_k, kv, T, H * 256, H * 256, 128) ||
        !make_rows_map(&tm_r, k_rope, T, kRopeDim, k_rope_row_stride, 128) || !make_rows_map(&tm_v, kv, T, H * 256, H * 256, 64))
        return CPA_ECUDA;
    if (plan->prefill_ctas < 1) return CPA_OK;
    latent_prefill_kernel<<<plan->prefill_ctas, kThreads, kPrefillSmem, (cudaStream_t)stream>>>(
        tm_q, tm_k, tm_r, tm_v, (__nv_bfloat16*)o, plan->dev(), (int)H, plan->q_tile, cfg->scale * 1.4426950408889634f,
        plan->prefill_rounds);
    return cudaGetLastError() == cudaSuccess ? CPA_OK : CPA_ECUDA;
}
