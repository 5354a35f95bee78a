// Latent rows into the paged cache: of a row x = [latent part | positional part],
//     c = x_c / sqrt(mean(x_c^2) + eps) * weight,      r = x_r turned to the token's position,
// in fp32, rounded once to bf16, to the token's slot and, where asked for, to a packed row.  Bound by memory: 2 (L + 64) bytes
// read and as many (or twice as many) written per token.  One warp takes a row: lane i holds the 16-byte pieces i, i + 32 and
// i + 64 of it, so the sum of squares is a warp's sum, and each lane computes one of the 32 sines and cosines.  Measured: 32 prompts
// of 1024..8192 tokens, latent parts of 512, packed rows as well, 473 MB, 77.5 us in a row = 93 % of the copy rate (78 to 83 by single
// calls); one row for each of 192 blocks 3.4 us on the device (latency).
#include <algorithm>

#include "latent.cuh"

namespace {

constexpr int kWarps = 8;

struct append_args {
    q8_tables t;
    const __nv_bfloat16* x;
    row_recipe recipe;
    const int32_t *cu, *first, *lens; // nullptr: one row per block; 0 everywhere; 0 everywhere
    int32_t* lens_out;
    __nv_bfloat16 *pool, *packed;
    int64_t x_row;
    int B, rows, row_ctas, at_once;
};

__device__ __forceinline__ int cu_at(const int32_t* cu, int b) { return cu ? ld_i32(cu + b) : b; }

// The last block that starts at or before a packed row, by a whole warp with 32 candidates per load.  What it leads to
// grows with the row, whatever cu holds.
__device__ __forceinline__ int find_block(int row, const int32_t* cu, int B, int lane) {
    if (!cu) return row;
    int lo = 0, size = B;
    while (size > 1) {
        const int step = (size + 31) / 32, i = lane * step;
        const uint32_t below = __ballot_sync(0xffffffffu, i < size && ld_i32(cu + lo + i) <= row);
        const int skip = max(__popc(below) - 1, 0) * step;
        lo += skip;
        size = min(step, size - skip);
    }
    return lo;
}

// A block's rows: n from packed row c0 on, to position `at`; and 0, or the status of why it is left out.
struct block_rows { int c0, n, at, ip, status; };
__device__ __forceinline__ block_rows rows_of(int b, const append_args& a) {
    const int c0 = cu_at(a.cu, b), c1 = cu_at(a.cu, b + 1), at = a.lens ? ld_i32(a.lens + b) : 0;
    const int ip = ld_i32(a.t.page_indptr + b), np = ld_i32(a.t.page_indptr + b + 1) - ip;
    const bool bad = c1 < c0 || at < 0 || c0 < 0 || c1 > a.rows;
    const int n = bad ? 0 : c1 - c0;
    return {c0, n, at, ip, bad ? kStatusInvalid : (int64_t)at + n > (int64_t)np * kPage ? kStatusNoSpace : 0};
}

// Packed row `row`, which is row `row - b.c0` of block b, through to its slot.
template <int L>
__device__ __forceinline__ void put_row(row_pieces<L>& r, int row, int block, const block_rows& b, const append_args& a, int lane) {
    const int at = b.at + row - b.c0;
    const int page = ld_i32(a.t.page_indices + b.ip + at / kPage);
    make_row<L>(r, a.recipe, (a.first ? ld_i32(a.first + block) : 0) + at, lane);
    store_row<L>(r, a.pool + ((int64_t)page * kPage + at % kPage) * (L + kRopeDim), lane);
    if (a.packed) store_row<L>(r, a.packed + (int64_t)row * (L + kRopeDim), lane);
}

// The block that the row warps take a row for.  The second row of a pair goes with the first one's block where it lies in that one's
// range, which is the block that its own search leads to as long as ranges run forwards.
__device__ __forceinline__ int taken_for(int row, const append_args& a, int lane) {
    if (a.at_once == 2 && (row & 1)) {
        const int b = find_block(row - 1, a.cu, a.B, lane);
        const block_rows o = rows_of(b, a);
        if (row >= o.c0 && row < o.c0 + o.n) return b;
    }
    return find_block(row, a.cu, a.B, lane);
}

template <int L, bool WIDE>
__global__ void __launch_bounds__(kWarps * 32) latent_append_kernel(const __grid_constant__ append_args a) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    row_pieces<L> r;
    if ((int)blockIdx.x >= a.row_ctas) {          // the blocks' books, a warp each
        for (int64_t b = (int64_t)((int)blockIdx.x - a.row_ctas) * kWarps + warp; b < a.B; b += (int64_t)(gridDim.x - a.row_ctas) * kWarps) {
            const block_rows o = rows_of((int)b, a);
            if (lane == 0) {
                if (o.status) atomicCAS(a.t.header, 0, o.status);
                if (a.lens_out) a.lens_out[b] = o.at + (o.status ? 0 : o.n);
            }
            if (o.status || o.n == 0 || !a.cu) continue;
            // Where a range runs backwards a good block's rows may be taken for others: those are taken here.  (What the search leads
            // to grows with the row, so a block's first and last one tell.)
            if (taken_for(o.c0, a, lane) == b && find_block(o.c0 + o.n - 1, a.cu, a.B, lane) == b) continue;
            for (int row = o.c0; row < o.c0 + o.n; ++row) {
                if (taken_for(row, a, lane) == b) continue;      // (x may hold the packed row by now)
                load_row<L, WIDE>(r, a.x + row * a.x_row, lane);
                put_row<L>(r, row, (int)b, o, a, lane);
            }
        }
        return;
    }
    // (where there are many rows a warp has two in flight, which mostly are the same block's: taken_for says for whom.  A search for the second
    // one as well in every pair cost 81 us for 78 on the prompts above.)
    row_pieces<L> r2;
    for (int64_t row = ((int64_t)blockIdx.x * kWarps + warp) * a.at_once; row < a.rows; row += (int64_t)a.row_ctas * kWarps * a.at_once) {
        const bool two = a.at_once == 2 && row + 1 < a.rows;
        load_row<L, WIDE>(r, a.x + row * a.x_row, lane);
        if (two) load_row<L, WIDE>(r2, a.x + (row + 1) * a.x_row, lane);
        int b = find_block((int)row, a.cu, a.B, lane);
        block_rows o = rows_of(b, a);
        if (!o.status && row >= o.c0 && row < o.c0 + o.n) put_row<L>(r, (int)row, b, o, a, lane);
        if (!two) continue;
        if (row + 1 >= o.c0 + o.n || row + 1 < o.c0) {
            b = find_block((int)row + 1, a.cu, a.B, lane);
            o = rows_of(b, a);
        }
        if (!o.status && row + 1 >= o.c0 && row + 1 < o.c0 + o.n) put_row<L>(r2, (int)row + 1, b, o, a, lane);
    }
}

template <int L>
int launch(const append_args& a, bool wide, int grid, cudaStream_t st) {
    return q8_launch(wide ? latent_append_kernel<L, true> : latent_append_kernel<L, false>, grid, kWarps * 32, st, a);
}

}  // namespace

extern "C" int cpa_latent_tables_config(const cpa_latent_config* cfg, cpa_config* out) {
    const int rc = latent_check(cfg);
    if (rc != CPA_OK || !out) return rc != CPA_OK ? rc : CPA_EINVAL;
    *out = latent_tables_cfg(*cfg);
    return CPA_OK;
}

extern "C" int cpa_latent_append(const cpa_latent_config* cfg, const cpa_table_dims* dims, void* d_tables,
                                 const cpa_rope_config* rope, const uint64_t* d_turns, const void* x, int64_t x_row_stride,
                                 const void* norm_weight, const int32_t* d_cu_new, int32_t num_rows, const int32_t* d_first,
                                 const int32_t* d_lens, int32_t* d_lens_out, void* pool, void* packed, void* stream) {
    int rc = latent_check(cfg);
    if (rc != CPA_OK) return rc;
    const cpa_config tc = latent_tables_cfg(*cfg);
    rc = q8_check(&tc, dims);
    if (rc != CPA_OK) return rc;
    const int row = cfg->latent_dim + kRopeDim;
    if (!d_tables || num_rows < 0 || (num_rows > 0 && !x) || !pool || !latent_aligned(d_tables, 16) || !latent_aligned(x, 2) ||
        !latent_aligned(norm_weight, 16) || !latent_aligned(pool, 16) || !latent_aligned(packed, 16) || !latent_aligned(d_turns, 8) ||
        !latent_aligned(d_cu_new, 4) || !latent_aligned(d_first, 4) || !latent_aligned(d_lens, 4) || !latent_aligned(d_lens_out, 4) ||
        (d_lens && d_lens == d_lens_out) || (d_turns != nullptr) != (rope != nullptr))
        return CPA_EINVAL;
    if (rope && (!rope_config_ok(rope) || rope->rope_dim != kRopeDim)) return CPA_EINVAL;
    if (!d_cu_new && num_rows != dims->num_blocks) return CPA_EINVAL;
    if (num_rows > 1 && (x_row_stride < row || (packed && packed == x && x_row_stride != row))) return CPA_EINVAL;
    append_args a = {};
    a.t = q8_view(tc, *dims, d_tables);
    a.x = (const __nv_bfloat16*)x;
    a.recipe = {(const __nv_bfloat16*)norm_weight, d_turns, cfg->norm_eps, rope ? (float)rope->amplitude : 1.f,
                rope && rope->layout == CPA_ROPE_INTERLEAVED};
    a.cu = d_cu_new;
    a.first = d_first;
    a.lens = d_lens;
    a.lens_out = d_lens_out;
    a.pool = (__nv_bfloat16*)pool;
    a.packed = (__nv_bfloat16*)packed;
    a.x_row = x_row_stride;
    a.B = dims->num_blocks;
    a.rows = num_rows;
    // two rows of a warp in flight where there are more than the device's warps (latent parts of 256: 6746 rows 5.1 us, 5.5 by one row
    // each; 11380 rows 6.9 and 7.5; below, 2116 rows 4.1 and 3.4)
    a.at_once = num_rows > 148 * 32 ? 2 : 1;
    a.row_ctas = (int)std::min<int64_t>(((int64_t)num_rows + kWarps * a.at_once - 1) / (kWarps * a.at_once), 1 << 20);
    const int grid = a.row_ctas + std::min((a.B + kWarps - 1) / kWarps, 1 << 16);
    const bool wide = latent_aligned(x, 16) && x_row_stride % 8 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    switch (cfg->latent_dim) {
        case 128: return launch<128>(a, wide, grid, st);
        case 256: return launch<256>(a, wide, grid, st);
        case 384: return launch<384>(a, wide, grid, st);
        default: return launch<512>(a, wide, grid, st);
    }
}
