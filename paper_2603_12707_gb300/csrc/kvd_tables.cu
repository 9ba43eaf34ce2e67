// kv_tables_step: block tables and slot map of a serving step, from request
// lengths that live on the device.
//
// Row r grows by n_r tokens from c_r: it needs u_r = ceil((c_r + n_r) / 16) -
// ceil(c_r / 16) pages.  With T_r and U_r the sums of max(n_i, 0) and u_i over
// rows i <= r, its tokens are T_r - n_r .. T_r - 1 of the packed batch, its
// pages entries U_r - u_r .. U_r - 1 of the free ring, and it is granted if
// T_r <= max_tokens and U_r <= free pages (or u_r = 0).  Rows that give tokens
// back are the same with a third sum.
#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kTablesThreads = 1024;
constexpr int kRowsPerThread = kKv4MaxBatch / kTablesThreads;

struct TablesArgs {
    int32_t* block_table;
    const int32_t* lens;
    int32_t* ring;
    const int32_t* state;
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
};

__device__ __forceinline__ int pages_of(int n) { return (n + kPageSize - 1) / kPageSize; }

// What the sums run over: tokens, pages taken, pages given back.
struct Sums {
    int64_t tokens, take, back;
};

__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b)
{
    return {a.tokens + b.tokens, a.take + b.take, a.back + b.back};
}

__device__ __forceinline__ Sums shift_up(const Sums& a, int n)
{
    return {__shfl_up_sync(0xffffffffu, a.tokens, n), __shfl_up_sync(0xffffffffu, a.take, n),
            __shfl_up_sync(0xffffffffu, a.back, n)};
}

// Exclusive sums over the block's threads, and the total.
__device__ Sums block_scan(const Sums& mine, Sums* total, Sums* warp_sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums s = mine;
    for (int n = 1; n < 32; n <<= 1) {
        const Sums o = shift_up(s, n);
        if (lane >= n) s = s + o;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    if (warp == 0) {
        Sums w = warp_sums[lane];
        for (int n = 1; n < 32; n <<= 1) {
            const Sums o = shift_up(w, n);
            if (lane >= n) w = w + o;
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    *total = warp_sums[31];
    const Sums before = warp > 0 ? warp_sums[warp - 1] : Sums{0, 0, 0};
    return {before.tokens + s.tokens - mine.tokens, before.take + s.take - mine.take, before.back + s.back - mine.back};
}

__global__ void __launch_bounds__(kTablesThreads) tables_kernel(TablesArgs a)
{
    __shared__ Sums warp_sums[32];
    __shared__ int32_t row_tok[kKv4MaxBatch];    // first token of each row (at most max_tokens)
    __shared__ int32_t row_page[kKv4MaxBatch];   // its first entry of the ring, -1: refused
    __shared__ int32_t row_seq[kKv4MaxBatch], row_len[kKv4MaxBatch];
    __shared__ unsigned long long taken;
    griddep_wait();
    griddep_launch_dependents();
    const int tid = threadIdx.x;
    if (tid == 0) taken = 0;

    int64_t head = a.state[0], count = a.state[1];
    if (head < 0 || head >= a.num_pages || count < 0 || count > a.num_pages) {
        if (tid == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
        head = count = 0;
    }
    if (a.lens_out != a.lens)
        for (int i = tid; i < a.max_seqs; i += kTablesThreads) a.lens_out[i] = a.lens[i];

    // The rows of this thread, consecutive ones.
    const int per = (a.batch + kTablesThreads - 1) / kTablesThreads;
    int seq[kRowsPerThread], ctx[kRowsPerThread], add[kRowsPerThread], take[kRowsPerThread], back[kRowsPerThread];
    bool fine[kRowsPerThread];
    Sums mine{0, 0, 0};
#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
        const int r = tid * per + k;
        seq[k] = ctx[k] = add[k] = take[k] = back[k] = 0;
        fine[k] = false;
        if (k >= per || r >= a.batch) continue;
        seq[k] = a.seq_ids ? a.seq_ids[r] : r;
        add[k] = a.new_lens[r];
        const bool known = seq[k] >= 0 && seq[k] < a.max_seqs;
        ctx[k] = known ? a.lens[seq[k]] : 0;
        const int64_t end = (int64_t)ctx[k] + add[k], most = (int64_t)a.max_pages * kPageSize;
        fine[k] = known && ctx[k] >= 0 && ctx[k] <= most && end >= 0 && end <= most;
        if (fine[k]) {
            const int d = pages_of((int)end) - pages_of(ctx[k]);
            take[k] = max(d, 0);
            back[k] = max(-d, 0);
        } else {
            kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
        }
        mine = mine + Sums{(int64_t)max(add[k], 0), take[k], back[k]};
    }
    Sums total;
    Sums at = block_scan(mine, &total, warp_sums);
    const bool fits = count + total.back <= a.num_pages;   // else a page has been given back twice
    if (!fits && tid == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
    if (a.lens_out != a.lens) __syncthreads();             // the copy above, before the changes below

#pragma unroll
    for (int k = 0; k < kRowsPerThread; ++k) {
        const int r = tid * per + k;
        if (k >= per || r >= a.batch) continue;
        const int grow = max(add[k], 0);
        const bool room = at.tokens + grow <= a.max_tokens || grow == 0;
        const bool paid = take[k] == 0 || at.take + take[k] <= count;
        const bool ok = fine[k] && room && paid && (fits || add[k] >= 0);
        if (fine[k] && !room) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
        if (fine[k] && room && !paid) kv4_error(a.err, KVC_DEVERR_OOM);
        row_tok[r] = (int32_t)min(at.tokens, (int64_t)a.max_tokens);
        row_page[r] = ok ? (int32_t)at.take : -1;
        row_seq[r] = seq[k];
        row_len[r] = ctx[k];
        if (a.cu) a.cu[r] = (int32_t)min(at.tokens, (int64_t)INT32_MAX);
        if (ok) {
            a.lens_out[seq[k]] = ctx[k] + add[k];
            if (take[k]) atomicMax(&taken, (unsigned long long)(at.take + take[k]));
            for (int i = 0; i < back[k]; ++i) {
                const int32_t page = a.block_table[(int64_t)seq[k] * a.max_pages + pages_of(ctx[k] + add[k]) + i];
                a.ring[(head + count + at.back + i) % a.num_pages] = page;
            }
        }
        at = at + Sums{(int64_t)grow, take[k], back[k]};
    }
    __syncthreads();
    if (tid == 0) {
        if (a.cu) a.cu[a.batch] = (int32_t)min(total.tokens, (int64_t)INT32_MAX);
        a.state_out[0] = (int32_t)((head + (int64_t)taken) % a.num_pages);
        a.state_out[1] = (int32_t)(count - (int64_t)taken + (fits ? total.back : 0));
    }

    // Tokens: the last row that starts at or before token t and is not empty holds it.
    const int64_t live = min(total.tokens, (int64_t)a.max_tokens);
    for (int64_t t = tid; t < a.max_tokens; t += kTablesThreads) {
        int64_t slot = -1;
        int pos = -1;
        if (t < live) {
            int lo = 0, hi = a.batch;   // first row that starts past t
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (row_tok[mid] <= t) lo = mid + 1;
                else hi = mid;
            }
            const int r = lo - 1;
            if (row_page[r] >= 0) {
                pos = row_len[r] + (int)(t - row_tok[r]);
                const int col = pos / kPageSize, fresh = col - pages_of(row_len[r]);
                int32_t* entry = a.block_table + (int64_t)row_seq[r] * a.max_pages + col;
                int32_t page;
                if (fresh >= 0) {
                    page = a.ring[(head + row_page[r] + fresh) % a.num_pages];
                    if (pos % kPageSize == 0) *entry = page;   // the token that opens the page
                } else {
                    page = *entry;
                }
                if (page >= 0 && page < a.num_pages) slot = (int64_t)page * kPageSize + pos % kPageSize;
                else kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
            }
        }
        a.slots[t] = slot;
        if (a.positions) a.positions[t] = pos;
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
    return kv4_launch_result(
        kv4_launch(tables_kernel, dim3(1), kTablesThreads, 0, static_cast<cudaStream_t>(stream), a));
}
