// Quantising append into the 8-bit cache, and rows of it read back as bf16.
//
// Append: per page, kv head and K or V, s = 2^e with amax(page) <= 448 s, code = e4m3(x / s); a page that holds tokens
// already keeps its scale or, when the new rows need a larger one, has its codes re-rounded (code * s_old / s_new).
// Read: bf16(code * s).  Both move 3 bytes per element (bf16 and code) and compute little, so HBM bounds them.  The
// unit of work is a touched (page, kv head) of K or of V: one warp takes all of it, because a scale needs the page's whole
// amax before the first code can be written; with the rows in registers everything is read once.  (K and V in one warp
// needs twice the registers and was slower.)  Consecutive warps take the heads of one page, so that a token's row is
// read whole.
//
// Units of work without a host that knows the lengths: block b is given the unit numbers from base_b = cu[b] / 16 + 2 b
// on.  n new tokens behind c cached ones touch at most n / 16 + 2 pages and base grows by at least that much, so the
// numbers never overlap and a unit finds its block by a search over cu alone; the few numbers left over do nothing.
// That holds while no range runs backwards.  Where one does, the search may lead from a good block's number elsewhere;
// so the warps that keep the blocks' books, one per block, look whether it does (the search's candidates are the same for
// every number, so a warp can tell for all pages of its block) and take those pages.  The books have CTAs of their own
// behind those of the units: in the units' loop they cost it registers (whole prompts 151 us, and 160 as a function that
// is not inlined, for 145).
//
// Measured: 32 prompts of 1024 .. 8192 tokens (8 heads of 128, 941 MB) 145 us = 6.5 TB/s, the card's copy rate; 8 blocks
// of 4096 tokens read back (201 MB) 34 us = 5.9 TB/s.
#include <algorithm>

#include "cache_q8.cuh"

namespace {

constexpr int kWarps = 8;

struct page_unit {
    int block;        // -1: nothing to do
    int page;         // pool page
    int p0, p1;       // its slots [p0, p1) are the new (or read) ones
    int row;          // packed row of slot p0
};

// cu == nullptr: one row per block
__device__ __forceinline__ int cu_at(const int32_t* cu, int b) { return cu ? ld_i32(cu + b) : b; }

// By a whole warp: 32 candidates are looked at per load.
__device__ __forceinline__ page_unit find_unit(int u, const q8_tables& t, const int32_t* cu, const int32_t* first, int B, int rows,
                                               int lane) {
    int lo = 0, size = B;
    while (size > 1) {
        const int step = (size + 31) / 32, i = lane * step, b = lo + i;
        const uint32_t below = __ballot_sync(0xffffffffu, i < size && cu_at(cu, b) / kPage + 2 * b <= u);
        const int skip = max(__popc(below) - 1, 0) * step;
        lo += skip;
        size = min(step, size - skip);
    }
    page_unit r{-1, 0, 0, 0, 0};
    const int c0 = cu_at(cu, lo), c1 = cu_at(cu, lo + 1), at = first ? ld_i32(first + lo) : 0;
    const int ip = ld_i32(t.page_indptr + lo), np = ld_i32(t.page_indptr + lo + 1) - ip;
    const int n = c1 - c0, j = u - (c0 / kPage + 2 * lo);
    if (n <= 0 || at < 0 || c0 < 0 || c1 > rows || j < 0) return r;
    if ((int64_t)at + n > (int64_t)np * kPage) return r;            // does not fit: the whole block is left out
    const int pg = at / kPage + j;
    if (pg * kPage >= at + n) return r;
    r.block = lo;
    r.page = ld_i32(t.page_indices + ip + pg);
    r.p0 = max(at - pg * kPage, 0);
    r.p1 = min(at + n - pg * kPage, kPage);
    r.row = c0 + pg * kPage + r.p0 - at;
    return r;
}

// A block's range of rows: n from packed row c0 on, to (or from) position `at`; and 0, or the status of why it is left out.
struct block_rows { int c0, n, at, ip, status; };

__device__ __forceinline__ block_rows rows_of(int b, const q8_tables& t, const int32_t* cu, const int32_t* first, int rows) {
    const int c0 = cu_at(cu, b), c1 = cu_at(cu, b + 1), at = first ? ld_i32(first + b) : 0;
    const int ip = ld_i32(t.page_indptr + b), np = ld_i32(t.page_indptr + b + 1) - ip;
    const bool bad = c1 < c0 || at < 0 || c0 < 0 || c1 > rows;
    const int n = bad ? 0 : c1 - c0;
    return {c0, n, at, ip, bad ? kStatusInvalid : (int64_t)at + n > (int64_t)np * kPage ? kStatusNoSpace : 0};
}

// Calls take(unit) for the pages of good block b whose unit numbers the search leads elsewhere (none, unless a range runs
// backwards), by a whole warp.
template <class F>
__device__ __forceinline__ void stray_units(int b, const block_rows& r, const q8_tables& t, const int32_t* cu, int B, int lane,
                                            F&& take) {
    constexpr int kLevels = 4;                    // of the search: 32^4 blocks
    static_assert(kMaxTableBlocks <= 1 << (5 * kLevels), "");
    // the candidates on the search's way to b: the first unit number of this lane's, and which one leads on
    int base[kLevels], on[kLevels], lo = 0, size = B;
#pragma unroll
    for (int l = 0; l < kLevels; ++l) {
        base[l] = INT32_MAX;
        on[l] = 0;
        if (size <= 1) continue;
        const int step = (size + 31) / 32, i = lane * step;
        if (i < size) base[l] = cu_at(cu, lo + i) / kPage + 2 * (lo + i);
        on[l] = (b - lo) / step;
        lo += on[l] * step;
        size = min(step, size - on[l] * step);
    }
    auto led_here = [&](int u) {
        bool yes = true;
#pragma unroll
        for (int l = 0; l < kLevels; ++l)
            yes = yes && max(__popc(__ballot_sync(0xffffffffu, base[l] <= u)) - 1, 0) == on[l];
        return yes;
    };
    const int page0 = r.at / kPage, pages = (r.at + r.n - 1) / kPage - page0 + 1, u0 = r.c0 / kPage + 2 * b;
    // (a candidate count grows with the number: what holds for the first and the last holds between them)
    if (led_here(u0) && led_here(u0 + pages - 1)) return;
    for (int j = 0; j < pages; ++j) {
        if (led_here(u0 + j)) continue;
        const int pg = page0 + j, p0 = max(r.at - pg * kPage, 0);
        take(page_unit{b, ld_i32(t.page_indices + r.ip + pg), p0, min(r.at + r.n - pg * kPage, kPage), r.c0 + pg * kPage + p0 - r.at});
    }
}

// The new rows of one unit, by a warp.
template <int D>
__device__ __forceinline__ void append_unit(const page_unit& u, int g, int kind, const uint4* k_new, const uint4* v_new,
                                            uint8_t* pool, float* scales, int Hkv, int lane) {
    constexpr int PIECES = D / 8;                 // 16-byte pieces of a bf16 row
    constexpr int N = kPage * PIECES / 32;        // pieces per lane of a page's K or V
    // this lane's piece of slots lane / PIECES + i * 32 / PIECES: 32 * Hkv pieces apart in the packed rows
    const int slot0 = lane / PIECES, piece = lane % PIECES;
    const uint4* from = (kind ? v_new : k_new) + (((int64_t)u.row + slot0 - u.p0) * Hkv + g) * PIECES + piece;
    uint4 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int slot = slot0 + i * (32 / PIECES);
        x[i] = slot >= u.p0 && slot < u.p1 ? __ldcs(from + i * (32 * Hkv)) : make_uint4(0, 0, 0, 0);
    }
    const int64_t cell = (int64_t)u.page * Hkv + g;
    float* sc = scales + cell * 2 + kind;
    uint8_t* to = pool + cell * (2 * kPage * D) + kind * (kPage * D);
    const float old = u.p0 > 0 ? ld_f32(sc) : 0.f;   // the page holds tokens already
    // largest magnitude, as bf16 bits of two halves; infinities and NaN, which do not count, are sorted out only
    // where the page has any
    uint32_t two = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
        two = __vmaxu2(__vmaxu2(two, __vmaxu2(x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu)),
                       __vmaxu2(x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu));
    uint32_t amax = __reduce_max_sync(0xffffffffu, max(two & 0xFFFFu, two >> 16)) << 16;
    if (amax >= 0x7F800000u) {
        amax = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) amax = max(amax, q8_amax8(x[i]));
        amax = __reduce_max_sync(0xffffffffu, amax);
    }
    float s = q8_scale(amax);
    if (u.p0 > 0) {
        if (s > old) {
            const float f = mul_keep(old, q8_inverse(s));   // (another writer's scale may be subnormal)
            for (int i = lane; i < u.p0 * (D / 4); i += 32) {
                uint32_t* c = reinterpret_cast<uint32_t*>(to) + i;
                *c = q8_rescale4(*c, f);
            }
        } else {
            s = old;
        }
    }
    uint8_t* dst = to + lane * 8;
    if (q8_power_of_two(s)) {
        const uint32_t inv = __float_as_uint(q8_inverse(s)), inv2 = inv | inv >> 16;      // a bf16 pair
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int slot = slot0 + i * (32 / PIECES);
            if (slot >= u.p0 && slot < u.p1) *reinterpret_cast<uint2*>(dst + i * 256) = q8_codes8_pow2(x[i], inv2);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int slot = slot0 + i * (32 / PIECES);
            if (slot >= u.p0 && slot < u.p1) *reinterpret_cast<uint2*>(dst + i * 256) = q8_codes8(x[i], s);
        }
    }
    __syncwarp();                             // every lane has read the old scale
    if (lane == 0) *sc = s;
}

// The books of block b, by a warp: its status and new length, and its stray pages.
template <int D>
__device__ __forceinline__ void append_books(int b, const q8_tables& t, const uint4* k_new, const uint4* v_new, const int32_t* cu,
                                             const int32_t* lens, int32_t* lens_out, uint8_t* pool, float* scales, int B,
                                             int rows, int Hkv, int lane) {
    const block_rows r = rows_of(b, t, cu, lens, rows);
    if (lane == 0) {
        if (r.status) atomicCAS(t.header, 0, r.status);
        if (lens_out) lens_out[b] = r.at + (r.status ? 0 : r.n);
    }
    if (r.status || r.n == 0) return;
    stray_units(b, r, t, cu, B, lane, [&](const page_unit& u) {
        for (int i = 0; i < 2 * Hkv; ++i) append_unit<D>(u, i >> 1, i & 1, k_new, v_new, pool, scales, Hkv, lane);
    });
}

// (four CTAs per SM: what hides the latency of the unit search and the loads is the number of warps; three, at the 74
// registers that the compiler would take, run at 154 us instead of 145 for 32 prompts of 1024 .. 8192 tokens)
template <int D>
__global__ void __launch_bounds__(kWarps * 32, 4)
kv_append_q8_kernel(q8_tables t, const uint4* k_new, const uint4* v_new, const int32_t* cu, const int32_t* lens,
                    int32_t* lens_out, uint8_t* pool, float* scales, int B, int rows, int Hkv, int64_t n_items, int item_ctas) {
    const int lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int warp = threadIdx.x >> 5;
    if ((int)blockIdx.x >= item_ctas) {           // the books
        for (int b = ((int)blockIdx.x - item_ctas) * kWarps + warp; b < B; b += ((int)gridDim.x - item_ctas) * kWarps)
            append_books<D>(b, t, k_new, v_new, cu, lens, lens_out, pool, scales, B, rows, Hkv, lane);
        return;
    }
    for (int64_t item = (int64_t)blockIdx.x * kWarps + warp; item < n_items; item += (int64_t)item_ctas * kWarps) {
        const int kind = (int)(item & 1), g = (int)((item >> 1) % Hkv);
        const page_unit u = find_unit((int)((item >> 1) / Hkv), t, cu, lens, B, rows, lane);
        if (u.block >= 0) append_unit<D>(u, g, kind, k_new, v_new, pool, scales, Hkv, lane);
    }
}

// The rows of one unit, by a warp.
template <int D>
__device__ __forceinline__ void read_unit(const page_unit& u, int g, int kind, const uint8_t* pool, const float* scales,
                                          uint4* k_out, uint4* v_out, int Hkv, int lane) {
    constexpr int PIECES = D / 8;                 // pieces of 8 codes of a row: a warp's stores are whole lines
    constexpr int N = kPage * PIECES / 32;        // pieces per lane of a page's K or V
    const int64_t cell = (int64_t)u.page * Hkv + g;
    const uint2* chunk = reinterpret_cast<const uint2*>(pool + cell * (2 * kPage * D) + kind * (kPage * D));
    const float s = ld_f32(scales + cell * 2 + kind);
    uint2 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int at = lane + 32 * i, slot = at / PIECES;
        x[i] = slot >= u.p0 && slot < u.p1 ? __ldcs(chunk + at) : make_uint2(0, 0);
    }
    uint4* out = (kind ? v_out : k_out) + ((int64_t)u.row * Hkv + g) * PIECES;
    auto two = [&](uint32_t codes) {
        const float2 f = e4m3x2_to_f32((uint16_t)codes);
        const __nv_bfloat162 r = __floats2bfloat162_rn(mul_keep(f.x, s), mul_keep(f.y, s));
        return *reinterpret_cast<const uint32_t*>(&r);
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int slot = (lane + 32 * i) / PIECES, piece = lane % PIECES;
        if (slot >= u.p0 && slot < u.p1)
            __stcs(out + (int64_t)(slot - u.p0) * Hkv * PIECES + piece,
                   make_uint4(two(x[i].x), two(x[i].x >> 16), two(x[i].y), two(x[i].y >> 16)));
    }
}

// The books of block b, as in the append.
template <int D>
__device__ __forceinline__ void read_books(int b, const q8_tables& t, const int32_t* cu, const int32_t* first, const uint8_t* pool,
                                           const float* scales, uint4* k_out, uint4* v_out, int B, int rows, int Hkv, int lane) {
    const block_rows r = rows_of(b, t, cu, first, rows);
    if (lane == 0 && r.status) atomicCAS(t.header, 0, r.status);
    if (r.status || r.n == 0) return;
    stray_units(b, r, t, cu, B, lane, [&](const page_unit& u) {
        for (int i = 0; i < 2 * Hkv; ++i) read_unit<D>(u, i >> 1, i & 1, pool, scales, k_out, v_out, Hkv, lane);
    });
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 5)
kv_read_q8_kernel(q8_tables t, const int32_t* cu, const int32_t* first, const uint8_t* pool, const float* scales, uint4* k_out,
                  uint4* v_out, int B, int rows, int Hkv, int64_t n_items, int item_ctas) {
    const int lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int warp = threadIdx.x >> 5;
    if ((int)blockIdx.x >= item_ctas) {           // the books
        for (int b = ((int)blockIdx.x - item_ctas) * kWarps + warp; b < B; b += ((int)gridDim.x - item_ctas) * kWarps)
            read_books<D>(b, t, cu, first, pool, scales, k_out, v_out, B, rows, Hkv, lane);
        return;
    }
    for (int64_t item = (int64_t)blockIdx.x * kWarps + warp; item < n_items; item += (int64_t)item_ctas * kWarps) {
        const int kind = (int)(item & 1), g = (int)((item >> 1) % Hkv);
        const page_unit u = find_unit((int)((item >> 1) / Hkv), t, cu, first, B, rows, lane);
        if (u.block >= 0) read_unit<D>(u, g, kind, pool, scales, k_out, v_out, Hkv, lane);
    }
}

// (page, head, K or V) items of `rows` rows over B blocks, idle unit numbers included; the CTAs that take them, and those
// for the books behind them, with a warp per block
int64_t page_items(int64_t rows, int B, int Hkv) { return (rows / kPage + 2 * (int64_t)B) * Hkv * 2; }
int page_ctas(int64_t items) { return (int)std::min<int64_t>((items + kWarps - 1) / kWarps, 1 << 20); }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

extern "C" int cpa_kv_append_q8(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const void* k_new,
                                const void* v_new, const int32_t* d_cu_new, int32_t num_rows, const int32_t* d_lens,
                                int32_t* d_lens_out, void* kv_pool, float* kv_scales, void* stream) {
    const int rc = q8_check(cfg, dims);
    if (rc != CPA_OK) return rc;
    if (!d_tables || (num_rows > 0 && (!k_new || !v_new)) || !kv_pool || !kv_scales || num_rows < 0 || !cpa_aligned16(d_tables) ||
        !cpa_aligned16(k_new) || !cpa_aligned16(v_new) || !cpa_aligned16(kv_pool) || !cpa_aligned16(kv_scales) ||
        !aligned4(d_cu_new) || !aligned4(d_lens) || !aligned4(d_lens_out) || (d_lens && d_lens == d_lens_out))
        return CPA_EINVAL;
    if (!d_cu_new && num_rows != dims->num_blocks) return CPA_EINVAL;
    const q8_tables t = q8_view(*cfg, *dims, d_tables);
    const int B = dims->num_blocks, Hkv = cfg->num_kv_heads;
    const int64_t items = page_items(num_rows, B, Hkv);
    auto kernel = cfg->head_dim == 128 ? kv_append_q8_kernel<128> : kv_append_q8_kernel<64>;
    return q8_launch(kernel, page_ctas(items) + page_ctas(B), kWarps * 32, (cudaStream_t)stream, t, (const uint4*)k_new,
                     (const uint4*)v_new, d_cu_new, d_lens, d_lens_out, (uint8_t*)kv_pool, kv_scales, B, num_rows, Hkv, items,
                     page_ctas(items));
}

extern "C" int cpa_kv_read_q8(const cpa_config* cfg, const cpa_table_dims* dims, void* d_tables, const int32_t* d_first,
                              const int32_t* d_cu, int32_t num_rows, const void* kv_pool, const float* kv_scales,
                              void* k_out, void* v_out, void* stream) {
    const int rc = q8_check(cfg, dims);
    if (rc != CPA_OK) return rc;
    if (!d_tables || !d_cu || !kv_pool || !kv_scales || (num_rows > 0 && (!k_out || !v_out)) || num_rows < 0 || !cpa_aligned16(d_tables) ||
        !cpa_aligned16(kv_pool) || !cpa_aligned16(kv_scales) || !cpa_aligned16(k_out) || !cpa_aligned16(v_out) ||
        !aligned4(d_first) || !aligned4(d_cu))
        return CPA_EINVAL;
    const q8_tables t = q8_view(*cfg, *dims, d_tables);
    const int B = dims->num_blocks, Hkv = cfg->num_kv_heads;
    const int64_t items = page_items(num_rows, B, Hkv);
    auto kernel = cfg->head_dim == 128 ? kv_read_q8_kernel<128> : kv_read_q8_kernel<64>;
    return q8_launch(kernel, page_ctas(items) + page_ctas(B), kWarps * 32, (cudaStream_t)stream, t, d_cu, d_first,
                     (const uint8_t*)kv_pool, kv_scales, (uint4*)k_out, (uint4*)v_out, B, num_rows, Hkv, items, page_ctas(items));
}
