// kv_tables_step: block tables and slot map of a serving step, from request
// lengths that live on the device.
//
// Row r grows by n_r tokens from c_r: it needs u_r = ceil((c_r + n_r) / 16) -
// ceil(c_r / 16) pages.  With T_r and U_r the sums of max(n_i, 0) and u_i over
// rows i <= r, its tokens are T_r - n_r .. T_r - 1 of the packed batch, its
// pages entries U_r - u_r .. U_r - 1 of the free ring, and it is granted if
// T_r <= max_tokens and U_r <= free pages (or u_r = 0).  Rows that give tokens
// back are the same with a third sum.
//
// Every CTA reads all rows and forms the sums (a few loads and a scan; rows are
// few next to tokens) and then works out its own tokens, whose rows it
// finds by binary search, so the map takes one launch.  What the call
// updates (lengths, the ring's state, pages given back) is written by the last CTA that has
// read it: a counter in the tables' state, zero between calls.
//
// A small call is latency, and much of that the fetching of its instructions
// (every launch fetches them anew): loops stay rolled.  On the device, 32 rows
// that decode take 3.6 us, 157 mixed rows 5.1, 1500 prompts of 450K
// tokens 10.0 (5.7 MB; the scan over the rows, then for every token a search of its row,
// which starts at the thread's last one, a load of its page id, and two stores).
#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kMaxThreads = 1024;

struct TablesArgs {
    int32_t* block_table;
    const int32_t* lens;
    int32_t* ring;
    const int32_t* state;
    int32_t* arrivals;      // the state's counter
    int64_t num_pages;
    int32_t max_seqs, max_pages, batch, max_tokens;
    int32_t cta_tokens;     // tokens of a CTA
    const int32_t* seq_ids;
    const int32_t* new_lens;
    int64_t* slots;
    int32_t* positions;
    int32_t* cu;
    int32_t* lens_out;
    int32_t* state_out;
    int32_t* err;
};

__device__ __forceinline__ int pages_of(int n) { return (n + kPageSize - 1) / kPageSize; }

// What the sums run over: tokens; pages taken in the high, given back in the low half.
struct Sums {
    int64_t tokens;
    uint64_t pages;
    __device__ __forceinline__ uint32_t take() const { return (uint32_t)(pages >> 32); }
    __device__ __forceinline__ uint32_t back() const { return (uint32_t)pages; }
};

__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return {a.tokens + b.tokens, a.pages + b.pages}; }
__device__ __forceinline__ Sums operator-(const Sums& a, const Sums& b) { return {a.tokens - b.tokens, a.pages - b.pages}; }

// Exclusive sums over the block's threads on top of `before`, which moves on by their total.
__device__ __forceinline__ Sums block_scan(const Sums& mine, Sums* before, Sums* warp_sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    Sums s = mine, ahead = {0, 0}, total = {0, 0};
#pragma unroll 1
    for (int level = 0; level < 2; ++level) {   // over the lanes, over the warps
#pragma unroll 1
        for (int n = 1; n < 32; n <<= 1) {
            const Sums o = {__shfl_up_sync(0xffffffffu, s.tokens, n), __shfl_up_sync(0xffffffffu, s.pages, n)};
            if (lane >= n) s = s + o;
        }
        if (level == 0) {
            ahead = s - mine;
            if (lane == 31) warp_sums[warp] = s;
            __syncthreads();
            s = lane < warps ? warp_sums[lane] : Sums{0, 0};
        }
    }
    const int from = max(warp - 1, 0);
    const Sums w = {__shfl_sync(0xffffffffu, s.tokens, from), __shfl_sync(0xffffffffu, s.pages, from)};
    total = {__shfl_sync(0xffffffffu, s.tokens, 31), __shfl_sync(0xffffffffu, s.pages, 31)};
    const Sums start = *before;
    *before = start + total;
    return start + ahead + (warp ? w : Sums{0, 0});
}

// Row of entry x: the last row from `lo` on whose first entry is at or before
// it (not empty, where x is below the sum); first[lo] <= x.
__device__ __forceinline__ int find_row(const int32_t* first, int lo, int batch, int x)
{
    int step = 1;
#pragma unroll 1
    for (; lo + step < batch && first[lo + step] <= x; step *= 2) lo += step;
    int hi = min(lo + step, batch);
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kMaxThreads) tables_kernel(TablesArgs a)
{
    extern __shared__ int32_t rows[];            // per row:
    int32_t* const row_tok = rows;               // first token (at most max_tokens)
    int32_t* const row_page = row_tok + a.batch; // its first entry of the ring, -1: refused
    int32_t* const row_len = row_page + a.batch; // tokens before
    int32_t* const row_seq = row_len + a.batch;
    int32_t* const row_back = row_seq + a.batch; // first of the pages given back
    __shared__ Sums warp_sums[kMaxThreads / 32];
    __shared__ uint32_t taken;
    __shared__ int is_last;
    const int tid = threadIdx.x, threads = blockDim.x;
    const bool speaks = blockIdx.x == 0;         // one CTA reports what all find
    if (tid == 0) taken = 0;
    griddep_wait();
    griddep_launch_dependents();

    int64_t head = a.state[0], count = a.state[1];
    // Rows, a block's threads at a time; the next ones are loaded meanwhile.
    const int64_t most = (int64_t)a.max_pages * kPageSize;
    Sums total{0, 0};
    int32_t errors = 0;
    auto row_seq_of = [&](int r) { return r >= a.batch ? -1 : a.seq_ids ? a.seq_ids[r] : r; };
    auto row_len_of = [&](int seq) { return seq >= 0 && seq < a.max_seqs ? a.lens[seq] : -1; };
    int seq = row_seq_of(tid), add = tid < a.batch ? a.new_lens[tid] : 0, ctx = row_len_of(seq);
    if (head < 0 || head >= a.num_pages || count < 0 || count > a.num_pages) {
        errors = KVC_DEVERR_PAGE_RANGE;
        head = count = 0;
    }
#pragma unroll 1
    for (int r0 = 0; r0 < a.batch; r0 += threads) {
        const int r = r0 + tid, next = r + threads;
        const int next_seq = row_seq_of(next), next_add = next < a.batch ? a.new_lens[next] : 0;
        const int64_t end = (int64_t)ctx + add;
        const bool fine = ctx >= 0 && ctx <= most && end >= 0 && end <= most;
        const int d = fine ? pages_of((int)end) - pages_of(ctx) : 0;
        const Sums mine = {max(add, 0), (uint64_t)max(d, 0) << 32 | (uint32_t)max(-d, 0)};
        const Sums at = block_scan(mine, &total, warp_sums);
        if (r < a.batch) {
            const bool room = at.tokens + mine.tokens <= a.max_tokens || mine.tokens == 0;
            const bool paid = mine.take() == 0 || (int64_t)at.take() + mine.take() <= count;
            const bool ok = fine && room && paid;
            if (!fine || !room) errors |= KVC_DEVERR_SEQ_RANGE;
            else if (!paid) errors |= KVC_DEVERR_OOM;
            row_tok[r] = (int32_t)min(at.tokens, (int64_t)a.max_tokens);
            row_page[r] = ok ? (int32_t)at.take() : -1;
            row_len[r] = ctx;
            row_seq[r] = seq;
            row_back[r] = (int32_t)at.back();
            if (ok && mine.take()) atomicMax(&taken, at.take() + mine.take());
            if (speaks && a.cu) a.cu[r] = (int32_t)min(at.tokens, (int64_t)INT32_MAX);
        }
        seq = next_seq;
        add = next_add;
        ctx = row_len_of(seq);
        __syncthreads();
    }
    const bool fits = count + total.back() <= a.num_pages;   // else a page has been given back twice
    if (!fits) errors |= KVC_DEVERR_PAGE_RANGE;
    if (errors && speaks) kv4_error(a.err, errors);
    // Every thread of this CTA has read the state and the lengths.
    if (tid == 0) is_last = gridDim.x == 1 || atomicAdd(a.arrivals, 1) == (int)gridDim.x - 1;

    // This CTA's tokens.
    const int live = (int)min(total.tokens, (int64_t)a.max_tokens);
    const int64_t first = (int64_t)blockIdx.x * a.cta_tokens, stop = min(first + a.cta_tokens, (int64_t)a.max_tokens);
    int r = 0;
#pragma unroll 1
    for (int64_t t = first + tid; t < stop; t += threads) {
        int64_t slot = -1;
        int pos = -1;
        if (t < live) {
            r = find_row(row_tok, r, a.batch, (int)t);
            if (row_page[r] >= 0) {
                const int len = row_len[r];
                pos = len + ((int)t - row_tok[r]);
                const int col = pos / kPageSize, fresh = col - pages_of(len);
                int32_t* const entry = a.block_table + (int64_t)row_seq[r] * a.max_pages + col;
                int64_t from = head + row_page[r] + fresh;
                if (from >= a.num_pages) from -= a.num_pages;
                const int32_t page = fresh >= 0 ? a.ring[from] : *entry;
                if (fresh >= 0 && pos % kPageSize == 0) *entry = page;   // the token that opens the page
                if (page >= 0 && page < a.num_pages) slot = (int64_t)page * kPageSize + pos % kPageSize;
                else kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
            }
        }
        a.slots[t] = slot;
        if (a.positions) a.positions[t] = pos;
    }
    __syncthreads();
    if (!is_last) return;

    // What the call updates, by the CTA that came last to reading it.
    if (a.lens_out != a.lens) {
#pragma unroll 1
        for (int i = tid; i < a.max_seqs; i += threads) a.lens_out[i] = a.lens[i];
        __syncthreads();
    }
#pragma unroll 1
    for (int i = tid; i < a.batch; i += threads) {
        const int n = a.new_lens[i];
        if (row_page[i] >= 0 && (fits || n >= 0)) a.lens_out[row_seq[i]] = row_len[i] + n;
    }
    // The k-th page given back: from its row's first page that is not needed any more.
    // Ids outside the pool are left out: where there are any, one warp does it again, and those behind move up.
    const int total_back = fits ? (int)total.back() : 0;
    int back = total_back, workers = threads;
    bool bad = false;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
        int given = 0;
        r = 0;
#pragma unroll 1
        for (int k0 = 0; k0 < total_back; k0 += workers) {
            const int k = k0 + tid;
            int32_t page = -1;
            if (k < total_back) {
                r = find_row(row_back, r, a.batch, k);
                const int kept = pages_of(row_len[r] + a.new_lens[r]);
                page = a.block_table[(int64_t)row_seq[r] * a.max_pages + kept + (k - row_back[r])];
            }
            const bool fine = page >= 0 && page < a.num_pages;
            bad |= !fine && k < total_back;
            int at = k;
            if (pass == 1) {
                const uint32_t some = __ballot_sync(0xffffffffu, fine);
                at = given + __popc(some & ((1u << tid) - 1u));
                given += __popc(some);
            }
            int64_t to = head + count + at;
            if (to >= a.num_pages) to -= a.num_pages;
            if (fine) a.ring[to] = page;
        }
        if (pass == 1) {
            back = given;
            break;
        }
        if (!__syncthreads_or(bad)) break;
        if (tid == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
        if (tid >= 32) return;
        workers = 32;
    }
    if (tid == 0) {
        if (a.cu) a.cu[a.batch] = (int32_t)min(total.tokens, (int64_t)INT32_MAX);
        int64_t next = head + taken;
        if (next >= a.num_pages) next -= a.num_pages;
        a.state_out[0] = (int32_t)next;
        a.state_out[1] = (int32_t)(count - taken + back);
        *a.arrivals = 0;
    }
}

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int kv_tables_step(const kv_tables* tables, int32_t batch, const int32_t* seq_ids,
                                      const int32_t* new_lens, int32_t max_tokens, int64_t* slots, int32_t* positions,
                                      int32_t* cu_seqlens, int32_t* lens_out, int32_t* free_state_out,
                                      int32_t* device_error, void* stream)
{
    if (int rc = kv4_check_tables(tables)) return rc;
    if (!tables->free_ring || !tables->free_state || !new_lens)
        return kv4_fail(KVC_ERR_INVALID, "kv_tables_step: null argument");
    if (tables->num_pages < 1 || tables->num_pages >= (int64_t)1 << 31)
        return kv4_fail(KVC_ERR_INVALID, "kv_tables_step: num_pages must be in 1 .. 2^31 - 1");
    if (batch < 1 || batch > kKv4MaxBatch) return kv4_fail(KVC_ERR_INVALID, "kv_tables_step: batch must be in 1 .. 4096");
    if (!seq_ids && batch > tables->max_seqs)
        return kv4_fail(KVC_ERR_INVALID, "kv_tables_step: more rows than requests, and no seq_ids");
    if (max_tokens < 0 || (max_tokens > 0 && !slots))
        return kv4_fail(KVC_ERR_INVALID, "kv_tables_step: max_tokens must be >= 0, with slots for them");
    TablesArgs a{};
    a.block_table = tables->block_table;
    a.lens = tables->lens;
    a.ring = tables->free_ring;
    a.state = tables->free_state;
    a.arrivals = tables->free_state + 2;
    a.num_pages = tables->num_pages;
    a.max_seqs = tables->max_seqs;
    a.max_pages = tables->max_pages;
    a.batch = batch;
    a.max_tokens = max_tokens;
    a.seq_ids = seq_ids;
    a.new_lens = new_lens;
    a.slots = slots;
    a.positions = positions;
    a.cu = cu_seqlens;
    a.lens_out = lens_out ? lens_out : tables->lens;
    a.state_out = free_state_out ? free_state_out : tables->free_state;
    a.err = device_error;
    static OncePerDevice once;
    constexpr int kRowBytes = 5 * (int)sizeof(int32_t);
    if (cudaError_t e = once.set_attribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowBytes * kKv4MaxBatch);
        e != cudaSuccess)
        return kv4_launch_result(e);
    // Few rows: small blocks, whose scans and barriers are shorter.  A CTA for
    // every two tokens of each thread, up to one per SM (every one reads all rows).
    const int threads = batch <= 256 ? 256 : kMaxThreads;
    int64_t ctas = ((int64_t)max_tokens + 2 * threads - 1) / (2 * threads);
    ctas = ctas < 1 ? 1 : ctas < 152 ? ctas : 152;
    a.cta_tokens = (int32_t)(((int64_t)max_tokens + ctas - 1) / ctas);
    return kv4_launch_result(kv4_launch(tables_kernel, dim3((unsigned)ctas), threads, (size_t)kRowBytes * batch,
                                        static_cast<cudaStream_t>(stream), a));
}
