// Block tables and slot maps built on the device from request lengths: the device counterpart of the index arrays that
// cpa_plan_create computes on the host, for lengths that only the device knows.
//
//   cu_seqlens[b+1]  = sum_{a<=b} L_a            page_indptr[b+1] = sum_{a<=b} ceil((L_a + T) / 16)
//   page list        = the first page_indptr[B] free pages (blocks take them in order)
//   slot(b, i)       = free[page_indptr[b] + i / 16] * 16 + i % 16
//
// The work is two prefix sums over B and a fill of the slot map: bytes are few (4 per token and page), so a call is
// bound by latency.  Hence one launch without any communication between its CTAs: every CTA sums all lengths (they come
// from L2, B words) and scans them chunk by chunk, and fills those tiles of the slot map that are its own.  (A second
// launch for the fill, or totals taken from the scan instead of a sum in front of it, have not been built.)
// 192 lengths, 147 k tokens: 5.3 us; 2000 lengths, 2.05 M tokens: 10.7 us (of which the sum and scan of 2000 lengths 3 us).
#include <algorithm>

#include "cache_q8.cuh"

namespace {

constexpr int kThreads = 512;
constexpr int kPerThread = 4;                     // blocks of a chunk per thread
constexpr int kChunk = kThreads * kPerThread;
constexpr int kRun = 8;                           // tokens per thread and tile of the fill
constexpr int kTile = kThreads * kRun;

struct pair64 { int64_t tokens, pages; };

// Sum over the CTA, given to every thread.
__device__ __forceinline__ pair64 cta_sum(pair64 v, pair64* sm) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.tokens += __shfl_xor_sync(0xffffffffu, v.tokens, o);
        v.pages += __shfl_xor_sync(0xffffffffu, v.pages, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    pair64 t{0, 0};
    for (int w = 0; w < kThreads / 32; ++w) { t.tokens += sm[w].tokens; t.pages += sm[w].pages; }
    return t;
}

__global__ void __launch_bounds__(kThreads)
tables_build_kernel(q8_tables t, const int32_t* lens, const int32_t* free_pages, int B, int T, int num_pages,
                    int page_limit, int token_limit, int n_tickets) {
    __shared__ int sm_cu[kChunk + 1], sm_ip[kChunk + 1];
    __shared__ pair64 sm_warp[kThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    // Totals, in 64 bits; a negative length or too many pages or tokens leaves empty tables and a status.  The lengths
    // of the first chunk stay in registers.
    // (this thread's first page id is fetched beside the first lengths, whether the blocks will take it or not)
    const int list0 = blockIdx.x * kThreads + tid;
    const int id0 = list0 < page_limit ? ld_i32(free_pages + list0) : 0;
    int L[kPerThread];
    pair64 sum{0, 0};
    bool bad = false;
    auto load = [&](int at) {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int b = at + tid * kPerThread + i;
            L[i] = b < B ? ld_i32(lens + b) : -1;
            bad |= b < B && L[i] < 0;
        }
    };
    auto pages_of = [&](int len) { return len < 0 ? 0 : (int)(((int64_t)len + T + kPage - 1) / kPage); };
    for (int at = (B - 1) / kChunk * kChunk; at >= 0; at -= kChunk) {
        load(at);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) { sum.tokens += max(L[i], 0); sum.pages += pages_of(L[i]); }
    }
    bad = __syncthreads_or((int)bad);
    const pair64 total = cta_sum(sum, sm_warp);
    const int32_t status = bad ? kStatusInvalid
                               : total.pages > page_limit || total.tokens > token_limit ? kStatusNoSpace : 0;
    for (int i = blockIdx.x * kThreads + tid; i < n_tickets; i += gridDim.x * kThreads) t.tickets[i] = 0;
    if (status) {
        for (int b = blockIdx.x * kThreads + tid; b <= B; b += gridDim.x * kThreads) t.cu_seqlens[b] = t.page_indptr[b] = 0;
        for (int i = tid; blockIdx.x == 0 && i < kHeaderWords; i += kThreads) t.header[i] = i == kBuildWords ? status : 0;
        return;
    }
    // every CTA writes its own word of the header, so nothing has to be cleared in front of the launch
    for (int i = tid; blockIdx.x == 0 && i < kHeaderWords; i += kThreads)
        if (i < kBuildWords || i >= kBuildWords + (int)gridDim.x)
            t.header[i] = i == 1 ? (int)total.tokens : i == 2 ? (int)total.pages : 0;

    pair64 run{0, 0};
    for (int at = 0; at < B; at += kChunk) {
        // exclusive scan of this chunk's lengths and pages on top of `run`
        if (at > 0) load(at);
        int tok[kPerThread], pg[kPerThread], mine_t = 0, mine_p = 0;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            tok[i] = mine_t;
            pg[i] = mine_p;
            mine_t += max(L[i], 0);
            mine_p += pages_of(L[i]);
        }
        int inc_t = mine_t, inc_p = mine_p;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int a = __shfl_up_sync(0xffffffffu, inc_t, o), c = __shfl_up_sync(0xffffffffu, inc_p, o);
            if (lane >= o) { inc_t += a; inc_p += c; }
        }
        __syncthreads();       // the previous chunk's fill and the totals are through with shared memory
        if (lane == 31) sm_warp[warp] = {inc_t, inc_p};
        __syncthreads();
        int base_t = (int)run.tokens, base_p = (int)run.pages;
        pair64 chunk{0, 0};
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) { base_t += (int)sm_warp[w].tokens; base_p += (int)sm_warp[w].pages; }
            chunk.tokens += sm_warp[w].tokens;
            chunk.pages += sm_warp[w].pages;
        }
        base_t += inc_t - mine_t;
        base_p += inc_p - mine_p;
        const int n = min(kChunk, B - at);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int j = tid * kPerThread + i;
            if (j > n) continue;
            sm_cu[j] = base_t + tok[i];
            sm_ip[j] = base_p + pg[i];
            if (blockIdx.x == 0 && j < n) { t.cu_seqlens[at + j] = sm_cu[j]; t.page_indptr[at + j] = sm_ip[j]; }
        }
        const int t0 = (int)run.tokens, t1 = (int)(run.tokens + chunk.tokens);
        run.tokens += chunk.tokens;
        run.pages += chunk.pages;
        if (tid == 0) { sm_cu[n] = t1; sm_ip[n] = (int)run.pages; }
        if (blockIdx.x == 0 && tid == 0 && at + n == B) { t.cu_seqlens[B] = t1; t.page_indptr[B] = (int)run.pages; }
        __syncthreads();
        if (t.slot_mapping == nullptr) continue;
        // Slots of the chunk's tokens, in tiles that go round the CTAs; a thread takes eight tokens (two 16-byte words of
        // the map), which mostly lie in one block and in one or two of its pages.
        const int grid = (int)gridDim.x, me = (int)blockIdx.x, from = t0 / kTile;
        for (int64_t tile = me + (from > me ? (from - me + grid - 1) / grid * grid : 0); tile * kTile < t1; tile += grid) {
            const int64_t g = tile * kTile + tid * kRun;
            const int first = (int)max((int64_t)t0, g), last = (int)min((int64_t)t1, g + kRun);
            if (first >= last) continue;
            int lo = 0, hi = n - 1;                                // last block of the chunk that starts at or before it
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (sm_cu[mid] <= first) lo = mid; else hi = mid - 1;
            }
            auto page_at = [&](int i) {
                const int page = ld_i32(free_pages + i);
                return (unsigned)page < (unsigned)num_pages ? page : 0;
            };
            if (last - first == kRun && sm_cu[lo + 1] >= last) {
                const int pos = first - sm_cu[lo], at = sm_ip[lo] + pos / kPage, off = pos % kPage;
                const int a = page_at(at), b = off + kRun > kPage ? page_at(at + 1) : a;
                int out[kRun];
#pragma unroll
                for (int i = 0; i < kRun; ++i) out[i] = (off + i < kPage ? a : b) * kPage + (off + i) % kPage;
#pragma unroll
                for (int i = 0; i < kRun; i += 4)
                    *reinterpret_cast<int4*>(t.slot_mapping + g + i) = make_int4(out[i], out[i + 1], out[i + 2], out[i + 3]);
            } else {
                for (int token = first; token < last; ++token) {
                    while (sm_cu[lo + 1] <= token) ++lo;           // blocks of length zero are stepped over
                    const int pos = token - sm_cu[lo];
                    t.slot_mapping[token] = page_at(sm_ip[lo] + pos / kPage) * kPage + pos % kPage;
                }
            }
        }
    }
    // the page list; an id outside the pool is replaced by page 0, so that no later call leaves the pool
    bool bad_id = false;
    for (int i = list0; i < (int)total.pages; i += gridDim.x * kThreads) {
        const int id = i == list0 ? id0 : ld_i32(free_pages + i);
        const bool out = (unsigned)id >= (unsigned)num_pages;
        bad_id |= out;
        t.page_indices[i] = out ? 0 : id;
    }
    bad_id = __syncthreads_or((int)bad_id);
    if (tid == 0) t.header[kBuildWords + blockIdx.x] = bad_id ? kStatusInvalid : 0;
}

}  // namespace

extern "C" int64_t cpa_tables_bytes(const cpa_config* cfg, const cpa_table_dims* dims) {
    const int rc = q8_check(cfg, dims);
    return rc != CPA_OK ? rc : q8_layout(*cfg, *dims).words * 4;
}

extern "C" int64_t cpa_tables_offset(const cpa_config* cfg, const cpa_table_dims* dims, int which) {
    const int rc = q8_check(cfg, dims);
    if (rc != CPA_OK) return rc;
    const q8_offsets o = q8_layout(*cfg, *dims);
    switch (which) {
        case CPA_ARR_CU_SEQLENS: return o.cu * 4;
        case CPA_ARR_PAGE_INDPTR: return o.indptr * 4;
        case CPA_ARR_PAGE_INDICES: return o.pages * 4;
        case CPA_ARR_SLOT_MAPPING: return o.slots * 4;
        default: return CPA_EINVAL;
    }
}

extern "C" int cpa_tables_build(const cpa_config* cfg, const cpa_table_dims* dims, const int32_t* d_block_lens,
                                const int32_t* d_free_pages, int32_t num_free, void* d_tables, void* stream) {
    const int rc = q8_check(cfg, dims);
    if (rc != CPA_OK) return rc;
    if (!d_block_lens || !d_free_pages || !d_tables || num_free < 0 || !cpa_aligned16(d_tables) ||
        (reinterpret_cast<uintptr_t>(d_block_lens) & 3u) || (reinterpret_cast<uintptr_t>(d_free_pages) & 3u))
        return CPA_EINVAL;
    q8_tables t = q8_view(*cfg, *dims, d_tables);
    if (dims->token_capacity == 0) t.slot_mapping = nullptr;
    const int page_limit = std::min(num_free, dims->page_capacity);
    const int token_limit = dims->token_capacity == 0 ? INT32_MAX : dims->token_capacity;
    cudaStream_t st = (cudaStream_t)stream;
    const int grid = std::max(1, std::min(kBuildCtas, (int)(std::max<int64_t>(dims->token_capacity, (int64_t)page_limit) / kTile) + 1));
    return q8_launch(tables_build_kernel, grid, kThreads, st, t, d_block_lens, d_free_pages, dims->num_blocks,
                     dims->max_new_tokens, dims->num_pages, page_limit, token_limit, dims->num_blocks * cfg->num_kv_heads);
}

extern "C" int cpa_tables_status(const void* d_tables, void* stream) {
    if (!d_tables) return CPA_EINVAL;
    int32_t head[kHeaderWords] = {};
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemcpyAsync(head, d_tables, sizeof(head), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) {
        (void)cudaGetLastError();
        return CPA_ECUDA;
    }
    int32_t word = head[0];
    for (int i = kBuildWords; i < kBuildWords + kBuildCtas; ++i)
        if (head[i]) word = head[i];          // faults of the build come first: what followed rests on them
    return word == 0 ? CPA_OK : word == kStatusNoSpace ? CPA_ENOSPC : word == kStatusInvalid ? CPA_EINVAL : CPA_ETIMEOUT;
}
