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
#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kTablesThreads = 512;
constexpr int kRowsPerThread = kKv4MaxBatch / kTablesThreads;
constexpr int kThreadTokens = 4;   // consecutive tokens of a thread: 16-byte stores
constexpr int kCtaTokens = kTablesThreads * kThreadTokens;

struct TablesArgs {
    int32_t* block_table;
    const int32_t* lens;
    int32_t* ring;
    const int32_t* state;
    int32_t* arrivals;      // the state's counter
    int64_t num_pages;
    int32_t max_seqs, max_pages, batch, max_tokens;
    const int32_t* seq_ids;
    const int32_t* new_lens;
    int64_t* slots;
    int32_t* positions;
    int32_t* cu;
    int32_t* lens_out;
    int32_t* state_out;
    int32_t* err;
    int32_t wide;           // slots and positions are 16-byte aligned
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

__device__ __forceinline__ Sums scan_warp(Sums s, int lane)
{
#pragma unroll
    for (int n = 1; n < 32; n <<= 1) {
        const Sums o = {__shfl_up_sync(0xffffffffu, s.tokens, n), __shfl_up_sync(0xffffffffu, s.pages, n)};
        if (lane >= n) s = s + o;
    }
    return s;
}

// Exclusive sums over the block's threads, and the total.
__device__ __forceinline__ Sums block_scan(const Sums& mine, Sums* total, Sums* warp_sums)
{
    constexpr int W = kTablesThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Sums s = scan_warp(mine, lane);
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    const Sums w = scan_warp(lane < W ? warp_sums[lane] : Sums{0, 0}, lane);
    const int from = warp > 0 ? warp - 1 : 0;
    Sums before = {__shfl_sync(0xffffffffu, w.tokens, from), __shfl_sync(0xffffffffu, w.pages, from)};
    if (warp == 0) before = {0, 0};
    *total = {__shfl_sync(0xffffffffu, w.tokens, W - 1), __shfl_sync(0xffffffffu, w.pages, W - 1)};
    return before + s - mine;
}

// Row of entry x: the last row whose first entry is at or before it (not empty, where x is below the sum).
__device__ __forceinline__ int find_row(const int32_t* first, int batch, int x)
{
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kTablesThreads) tables_kernel(TablesArgs a)
{
    extern __shared__ int32_t rows[];            // per row:
    int32_t* const row_tok = rows;               // first token (at most max_tokens)
    int32_t* const row_page = row_tok + a.batch; // its first entry of the ring, -1: refused
    int32_t* const row_len = row_page + a.batch; // tokens before
    int32_t* const row_seq = row_len + a.batch;
    int32_t* const row_back = row_seq + a.batch; // first of the pages given back
    __shared__ Sums warp_sums[kTablesThreads / 32];
    __shared__ uint32_t taken;
    __shared__ int is_last;
    griddep_wait();
    griddep_launch_dependents();
    const int tid = threadIdx.x;
    const bool speaks = blockIdx.x == 0;         // one CTA reports what all find
    if (tid == 0) taken = 0;

    int64_t head = a.state[0], count = a.state[1];
    if (head < 0 || head >= a.num_pages || count < 0 || count > a.num_pages) {
        if (tid == 0 && speaks) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
        head = count = 0;
    }

    // The rows of this thread, consecutive ones.
    const int per = (a.batch + kTablesThreads - 1) / kTablesThreads;
    const int64_t most = (int64_t)a.max_pages * kPageSize;
    int seq[kRowsPerThread], ctx[kRowsPerThread], add[kRowsPerThread];
    Sums of[kRowsPerThread], mine{0, 0};
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
        const int r = tid * per + k;
        seq[k] = -1;
        add[k] = 0;
        if (k < per && r < a.batch) {
            seq[k] = a.seq_ids ? a.seq_ids[r] : r;
            add[k] = a.new_lens[r];
        }
    }
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) ctx[k] = seq[k] >= 0 && seq[k] < a.max_seqs ? a.lens[seq[k]] : -1;
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
        const int64_t end = (int64_t)ctx[k] + add[k];
        const bool fine = ctx[k] >= 0 && ctx[k] <= most && end >= 0 && end <= most;
        const int d = fine ? pages_of((int)end) - pages_of(ctx[k]) : 0;
        of[k] = {max(add[k], 0), (uint64_t)max(d, 0) << 32 | (uint32_t)max(-d, 0)};
        if (!fine) ctx[k] = -1;
        mine = mine + of[k];
    }
    Sums total;
    Sums at = block_scan(mine, &total, warp_sums);
    const bool fits = count + total.back() <= a.num_pages;   // else a page has been given back twice
    if (!fits && tid == 0 && speaks) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);

    int32_t errors = 0;
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
        const int r = tid * per + k;
        if (k >= per || r >= a.batch) continue;
        const bool room = at.tokens + of[k].tokens <= a.max_tokens || of[k].tokens == 0;
        const bool paid = of[k].take() == 0 || (int64_t)at.take() + of[k].take() <= count;
        const bool ok = ctx[k] >= 0 && room && paid && (fits || add[k] >= 0);
        if (ctx[k] < 0 || !room) errors |= KVC_DEVERR_SEQ_RANGE;
        else if (!paid) errors |= KVC_DEVERR_OOM;
        row_tok[r] = (int32_t)min(at.tokens, (int64_t)a.max_tokens);
        row_page[r] = ok ? (int32_t)at.take() : -1;
        row_len[r] = ctx[k];
        row_seq[r] = seq[k];
        row_back[r] = (int32_t)at.back();
        if (ok && of[k].take()) atomicMax(&taken, at.take() + of[k].take());
        at = at + of[k];
    }
    if (errors && speaks) kv4_error(a.err, errors);
    __syncthreads();
    // Every thread of this CTA has read the state and the lengths.
    if (tid == 0) is_last = gridDim.x == 1 || atomicAdd(a.arrivals, 1) == (int)gridDim.x - 1;

    // Tokens.
    const int live = (int)min(total.tokens, (int64_t)a.max_tokens);
    for (int64_t t0 = ((int64_t)blockIdx.x * kTablesThreads + tid) * kThreadTokens; t0 < a.max_tokens;
         t0 += (int64_t)gridDim.x * kCtaTokens) {
        int64_t slot[kThreadTokens];
        int pos[kThreadTokens];
        int r = -1, stop = 0, col_now = -1;      // the row in work, its end, the page in hand
        int32_t page = -1;
#pragma unroll
        for (int k = 0; k < kThreadTokens; ++k) {
            const int t = (int)t0 + k;
            slot[k] = -1;
            pos[k] = -1;
            if (t >= live) continue;
            if (t >= stop) {
                r = r < 0 ? find_row(row_tok, a.batch, t) : r + 1;
                while (r + 1 < a.batch && row_tok[r + 1] <= t) ++r;
                stop = r + 1 < a.batch ? row_tok[r + 1] : live;
                col_now = -1;
            }
            if (row_page[r] < 0) continue;
            pos[k] = row_len[r] + (t - row_tok[r]);
            const int col = pos[k] / kPageSize, fresh = col - pages_of(row_len[r]);
            if (col != col_now) {
                int32_t* entry = a.block_table + (int64_t)row_seq[r] * a.max_pages + col;
                if (fresh >= 0) {
                    int64_t from = head + row_page[r] + fresh;
                    if (from >= a.num_pages) from -= a.num_pages;
                    page = a.ring[from];
                    if (pos[k] % kPageSize == 0) *entry = page;   // the token that opens the page
                } else {
                    page = *entry;
                }
                col_now = col;
                if (page < 0 || page >= a.num_pages) {
                    kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
                    page = -1;
                }
            }
            if (page >= 0) slot[k] = (int64_t)page * kPageSize + pos[k] % kPageSize;
        }
        if (a.wide && t0 + kThreadTokens <= a.max_tokens) {
            longlong2* to = reinterpret_cast<longlong2*>(a.slots + t0);
            to[0] = make_longlong2(slot[0], slot[1]);
            to[1] = make_longlong2(slot[2], slot[3]);
            if (a.positions) *reinterpret_cast<int4*>(a.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
#pragma unroll
            for (int k = 0; k < kThreadTokens; ++k)
                if (t0 + k < a.max_tokens) {
                    a.slots[t0 + k] = slot[k];
                    if (a.positions) a.positions[t0 + k] = pos[k];
                }
        }
    }
    __syncthreads();
    if (!is_last) return;

    // What the call updates, by the CTA that came last to reading it.
    if (a.lens_out != a.lens) {
        for (int i = tid; i < a.max_seqs; i += kTablesThreads) a.lens_out[i] = a.lens[i];
        __syncthreads();
    }
    at = at - mine;
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
        const int r = tid * per + k;
        if (k >= per || r >= a.batch) continue;
        if (a.cu) a.cu[r] = (int32_t)min(at.tokens, (int64_t)INT32_MAX);
        if (row_page[r] >= 0) a.lens_out[seq[k]] = ctx[k] + add[k];
        at = at + of[k];
    }
    // The k-th page given back: from its row's first page that is not needed any more.
    const int back = fits ? (int)total.back() : 0;
    for (int k = tid; k < back; k += kTablesThreads) {
        const int r = find_row(row_back, a.batch, k);
        const int kept = pages_of(row_len[r] + a.new_lens[r]);
        const int32_t page = a.block_table[(int64_t)row_seq[r] * a.max_pages + kept + (k - row_back[r])];
        int64_t to = head + count + k;
        if (to >= a.num_pages) to -= a.num_pages;
        a.ring[to] = page;
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
    a.wide = kv4_aligned(slots, 16) && kv4_aligned(positions, 16);
    static OncePerDevice once;
    constexpr int kRowBytes = 5 * (int)sizeof(int32_t);
    if (cudaError_t e = once.set_attribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowBytes * kKv4MaxBatch);
        e != cudaSuccess)
        return kv4_launch_result(e);
    // A CTA for every kCtaTokens tokens, up to one per SM (every one reads all rows).
    const int64_t ctas = ((int64_t)max_tokens + kCtaTokens - 1) / kCtaTokens;
    return kv4_launch_result(kv4_launch(tables_kernel, dim3((unsigned)(ctas < 1 ? 1 : ctas < 152 ? ctas : 152)), kTablesThreads,
                                        (size_t)kRowBytes * batch, static_cast<cudaStream_t>(stream), a));
}
