// kv16_plan: the plan of a decode step over shared prefixes (kvd_kv16_plan.h),
// made from the lengths on the device.  Every CTA finds the places of all rows and writes a part of the plan.  Runs of rows with one prefix come from a scan of maxima
// over their first rows, places in the two lines of work from scans of sums, each worker's start from a
// binary search.  Bound by latency: loads, two scans, searches and their instructions, fetched anew by each launch.
// 32 rows take 4.8 us, 150 rows in 11 groups 7.8 us, once a step for all its layers.
#include "kvd_kv16_plan.h"

namespace kvd {
namespace {

constexpr int kPlanMaxThreads = 512;

struct StepPlanArgs {
    PlanView view;
    const int32_t* lens;
    const int32_t* seq_ids;
    const int32_t* prefix_ids;
    int32_t max_seqs, max_pages;
    int32_t batch, hq, hkv, dim, grid;
    int32_t* err;
};

struct Sums {
    int64_t units, cost;
    int32_t cols, rows;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b)
{
    return {a.units + b.units, a.cost + b.cost, a.cols + b.cols, a.rows + b.rows};
}
__device__ __forceinline__ Sums shuffle_up(const Sums& s, int n)
{
    return {__shfl_up_sync(0xffffffffu, s.units, n), __shfl_up_sync(0xffffffffu, s.cost, n), __shfl_up_sync(0xffffffffu, s.cols, n),
            __shfl_up_sync(0xffffffffu, s.rows, n)};
}
__device__ __forceinline__ Sums broadcast(const Sums& s, int from)
{
    return {__shfl_sync(0xffffffffu, s.units, from), __shfl_sync(0xffffffffu, s.cost, from), __shfl_sync(0xffffffffu, s.cols, from),
            __shfl_sync(0xffffffffu, s.rows, from)};
}
struct Max {
    int32_t v;
};
__device__ __forceinline__ Max broadcast(const Max& s, int from) { return {__shfl_sync(0xffffffffu, s.v, from)}; }
__device__ __forceinline__ Max operator+(const Max& a, const Max& b) { return {max(a.v, b.v)}; }
__device__ __forceinline__ Max shuffle_up(const Max& s, int n) { return {__shfl_up_sync(0xffffffffu, s.v, n)}; }

// Inclusive scan over the block's threads on top of `before`, which moves on by the total.
// (By the first `warps` warps, which hold all rows; the others only keep the barriers.)
template <class S>
__device__ __forceinline__ S block_scan(S s, S* before, S* warp_sums, int warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (warp >= warps) {
        __syncthreads();
        __syncthreads();
        return s;
    }
#pragma unroll 1
    for (int n = 1; n < 32; n <<= 1) {
        const S o = shuffle_up(s, n);
        if (lane >= n) s = o + s;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    S t = warp_sums[lane < warps ? lane : warps - 1];
#pragma unroll 1
    for (int n = 1; n < warps; n <<= 1) {
        const S o = shuffle_up(t, n);
        if (lane >= n && lane < warps) t = o + t;
    }
    const S start = *before;
    s = start + s;
    const S ahead = broadcast(t, max(warp - 1, 0));
    if (warp > 0) s = ahead + s;
    *before = start + broadcast(t, warps - 1);
    __syncthreads();
    return s;
}

__device__ __forceinline__ int pages_of(int n) { return (n + kPageSize - 1) / kPageSize; }

// The last entry of first[0 .. n - 1] that is at or below x.
template <class I>
__device__ __forceinline__ int last_at(const I* first, int n, I x)
{
    int lo = 0, hi = n;
#pragma unroll 1
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Bytes of shared memory for each row.
constexpr int kPlanRowBytes = 8 + 12 * 4;

__global__ void __launch_bounds__(kPlanMaxThreads) plan_kernel(StepPlanArgs a)
{
    extern __shared__ int64_t shared[];
    const int B = a.batch;
    int64_t* const s_cost = shared;                                   // by row: first cost unit of the run that starts there
    int32_t* s_next = reinterpret_cast<int32_t*>(s_cost + B);
    auto take = [&](int n) {
        int32_t* const p = s_next;
        s_next += n * B;
        return p;
    };
    int32_t* const s_unit = take(2);     // by record: its first unit
    int32_t* const s_col = take(2);      // query rows before it
    int32_t* const s_req = take(1);      // the row's request
    int32_t* const s_len = take(1);      // and its tokens
    int32_t* const s_pre = take(1);      // prefix, -1: none, of length 0 or refused
    int32_t* const s_plen = take(1);     // its tokens
    int32_t* const s_rows = take(1);     // rows of the run that starts here
    int32_t* const s_first = take(1);    // first row of the run that the row is in
    int32_t* const s_before = take(1);   // rows in large runs before
    int32_t* const s_pages = take(1);    // of the run that starts here; 0: none does
    __shared__ PlanHeader s_header;
    __shared__ Sums sum_warps[kPlanMaxThreads / 32];
    __shared__ Max max_warps[kPlanMaxThreads / 32];
    const int tid = threadIdx.x, threads = blockDim.x, G = a.hq / a.hkv;
    const int warps_needed = min((B + 31) / 32, threads / 32);
    const bool speaks = blockIdx.x == 0;       // one CTA writes and reports what all find
    griddep_wait();
    griddep_launch_dependents();

    const int64_t most = (int64_t)a.max_pages * kPageSize;
    auto length = [&](int req, bool* bad) {
        if (req < 0 || req >= a.max_seqs) {
            *bad = true;
            return 0;
        }
        const int n = a.lens[req];
        if (n < 0 || n > most) {
            *bad = true;
            return 0;
        }
        return n;
    };
    bool any_bad = false;
#pragma unroll 1
    for (int r = tid; r < B; r += threads) {
        const int req = a.seq_ids ? a.seq_ids[r] : r, pre = a.prefix_ids ? a.prefix_ids[r] : -1;
        bool bad = false;
        const int n = length(req, &bad), np = pre == -1 ? 0 : length(pre, &bad);
        any_bad |= bad;
        s_req[r] = req;
        s_len[r] = bad ? 0 : n;
        s_pre[r] = bad || np == 0 ? -1 : pre;
        s_plen[r] = np;
    }
    if (any_bad && speaks) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
    __syncthreads();
    // Runs.
    Max before_max{-1};
#pragma unroll 1
    for (int r0 = 0; r0 < B; r0 += threads) {
        const int r = r0 + tid;
        const int pre = r < B ? s_pre[r] : -1;
        const bool starts = r < B && (r == 0 || s_pre[r - 1] != pre);
        const Max at = block_scan(Max{starts ? r : -1}, &before_max, max_warps, warps_needed);
        if (r < B) {
            s_first[r] = pre >= 0 ? at.v : -1;
            if (r + 1 == B || s_pre[r + 1] != pre) s_rows[at.v] = r + 1 - at.v;
        }
    }
    __syncthreads();
    // A run's chunks.
    auto chunks_of = [&](int rows) {
        const int pair = 2 * (kTileRows / G), each = chunk_rows(rows, (rows + pair - 1) / pair);
        return (rows + each - 1) / each;   // (nearly equal: the last ones might have been left without rows)
    };
    // Places in the lines of work.
    Sums total{0, 0, 0, 0};
#pragma unroll 1
    for (int r0 = 0; r0 < B; r0 += threads) {
        const int r = r0 + tid;
        Sums mine{0, 0, 0, 0};
        Run run{};
        int small_pages = 0, rows = 0, pages = 0;
        if (r < B) {
            if (s_first[r] == r) {
                rows = s_rows[r];
                pages = pages_of(s_plen[r]);
                if (rows * G <= kRecordCols) {
                    small_pages = pages;
                    mine.cols = rows * G;
                } else {
                    run.chunks = chunks_of(rows);
                    const int cost = page_cost(rows, run.chunks, G);
                    mine.cost = (int64_t)(pages + job_start(cost)) * a.hkv * run.chunks * cost;
                    mine.rows = rows;
                }
            }
            mine.units = (int64_t)(small_pages + pages_of(s_len[r])) * a.hkv;
            mine.cols += G;
        }
        const Sums at = block_scan(mine, &total, sum_warps, warps_needed);
        if (r < B) {
            const int64_t unit = at.units - mine.units;
            s_unit[2 * r] = (int32_t)unit;
            s_unit[2 * r + 1] = (int32_t)(unit + (int64_t)small_pages * a.hkv);
            s_col[2 * r] = at.cols - mine.cols;
            s_col[2 * r + 1] = at.cols - G;
            s_pages[r] = pages;
            s_cost[r] = at.cost - mine.cost;
            s_before[r] = at.rows - mine.rows;
            if (blockIdx.x == 1) {             // (others than the one that writes the header)
                run.req = s_pre[r];
                run.len = s_plen[r];
                run.pages = mine.cost ? pages : 0;
                run.rows = rows;
                run.cost = s_cost[r];
                run.rows_before = s_before[r];
                a.view.runs[r] = run;
            }
            if (blockIdx.x == 2) {
                const int n = s_len[r];
                a.view.recs[2 * r] = Record{s_pre[r], s_plen[r], small_pages, r, rows, s_unit[2 * r], s_col[2 * r], 0};
                a.view.recs[2 * r + 1] = Record{s_req[r], n, pages_of(n), r, 1, s_unit[2 * r + 1], s_col[2 * r + 1], 0};
            }
        }
    }
    __syncthreads();                       // (the search for the first large run below reads all rows' places)
    if (tid < 32) {
        // CTAs for large runs, the others for records: the cut at which the slower side is fastest.  (All lanes alike, but for the
        // shares, of which each other lane makes the other kind's.  Quotients are within two steps of 2^-24; 64-bit floating point is far slower.)
        const bool fits = total.units < (int64_t)1 << 31 && total.cost < (int64_t)1 << 40;
        int ctas = 0;
        if (total.cost > 0) {
            const float c = (float)total.cost, u = (float)total.units * record_cost(a.dim);
            ctas = a.grid;
            if (total.units > 0) {
                const int f = min(max((int)__fdividef(a.grid * c, c + u), 1), a.grid - 1), g = min(f + 1, a.grid - 1);
                ctas = max(__fdividef(c, (float)f), __fdividef(u, (float)(a.grid - f))) <= max(__fdividef(c, (float)g), __fdividef(u, (float)(a.grid - g))) ? f : g;
            }
            // One run whose rows come in chunks: the same number of CTAs for each of its jobs, so that the chunks' CTAs read the same
            // pages at about the same time, from L2 but for the first.
            if (total.rows * G > 2 * kTileRows) {
                const int r = last_at(s_cost, B, (int64_t)0), chunks = chunks_of(s_rows[r]), jobs = a.hkv * chunks;
                if (s_rows[r] == total.rows && chunks > 1 && ctas % jobs * 8 <= ctas) ctas -= ctas % jobs;
            }
            if (total.cost < (int64_t)ctas * kLeastRunPages * kWideCost) ctas = max((int)total.cost / (kLeastRunPages * kWideCost), 1);
        }
        if (!fits && speaks && tid == 0) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
        const int warps = (int)min((int64_t)(a.grid - ctas) * kAttnWarps, (total.units + kLeastRecordPages - 1) / kLeastRecordPages);
        if (tid < 2) {
            Shares shares{};
            if (fits) shares = make_shares(tid ? total.cost : total.units, tid ? ctas : warps);
            PlanHeader h{};
            h.magic = fits ? kPlanMagic : 0;
            h.batch = B;
            h.hq = a.hq;
            h.hkv = a.hkv;
            h.dim = a.dim;
            h.grid = a.grid;
            h.max_seqs = a.max_seqs;
            h.max_pages = a.max_pages;
            h.prefix_ctas = ctas;
            if (tid == 1) s_header.cost = shares;
            __syncwarp(3u);
            if (tid == 0) {
                h.units = shares;
                h.cost = s_header.cost;
                s_header = h;
                if (speaks) *a.view.header = h;
            }
        }
    }
    __syncthreads();
    if (s_header.magic == 0) return;
    // Where workers start, and what the merge reads of a row, by all CTAs' threads.
    const int all = threads * gridDim.x, at0 = blockIdx.x * threads + tid;
    const Shares units = s_header.units, costs = s_header.cost;
    // Workers of records lie over the CTAs by turns, so that few of them are on different SMs.
    const int rec_ctas = a.grid - costs.n;
#pragma unroll 1
    for (int i = at0; i < rec_ctas * kAttnWarps; i += all) {
        const int w = i, warp = w / rec_ctas, cta = costs.n + w - warp * rec_ctas;
        WarpStart* const to = &a.view.warp_starts[cta * kAttnWarps + warp];
        if (w >= units.n) {
            to->count = 0;
        } else {
            WarpStart x{};
            x.worker = w;
            const int32_t u = (int32_t)units.start(w);
            const int k = last_at(s_unit, 2 * B, u), r = k >> 1;
            const bool own = k & 1;
            const int len = own ? s_len[r] : s_plen[r], pages = pages_of(len), off = u - s_unit[k];
            x.rec = k;
            x.head = (int)divide(off, pages);
            x.page = off - x.head * pages;
            x.count = (int32_t)units.start(w + 1) - u;
            x.r = Record{own ? s_req[r] : s_pre[r], len, pages, r, own ? 1 : s_rows[r], s_unit[k], s_col[k], 0};
            *to = x;
        }
    }
#pragma unroll 1
    for (int c = all - 1 - at0; c < costs.n; c += all) {
        const int64_t at = costs.start(c), end = costs.start(c + 1);
        const int i = last_at(s_cost, B, at), rows = s_rows[i], chunks = chunks_of(rows);
        const Run run{s_pre[i], s_plen[i], s_pages[i], rows, s_cost[i], s_before[i], chunks};
        const int w = page_cost(rows, chunks, G), start = job_start(w);
        // The first page that starts at or after the share; the segment may be of the run's next job, or of none.
        const int64_t page = pages_at(at - run.cost, w);
        int job = (int)divide(page, run.pages + start), p = max((int)(page - (int64_t)job * (run.pages + start)) - start, 0);
        Segment s{};
        if (p < run.pages && job < chunks * a.hkv) s = make_segment(run, i, job, p, end, a.hkv, G, c);
        if (s.pages > 0 || p > 0) ++job;
        a.view.cta_starts[c] = CtaStart{i, job, end, run, s};
    }
#pragma unroll 1
    for (int i = at0 < all / 2 ? at0 + all / 2 : at0 - all / 2; i < B * a.hkv; i += all) {   // (other threads first)
        const int r = i / a.hkv, kv = i - r * a.hkv, first = s_first[r], pages = pages_of(s_len[r]);
        RowSources x{};
        auto segments = [](const Shares& s, int64_t u, int64_t last, int* w0) {
            *w0 = s.worker(u);
            return s.worker(last) - *w0 + 1;
        };
        int w0;
        if (pages > 0) {
            const int64_t u = (int64_t)s_unit[2 * r + 1] + (int64_t)kv * pages;
            x.own_count = segments(units, u, u + pages - 1, &w0);
            x.own = record_entry(s_col[2 * r + 1], 1, a.hkv, G, kv, w0);
        }
        if (first >= 0) {
            const int rows = s_rows[first], ppages = pages_of(s_plen[r]);
            if (rows * G <= kRecordCols) {
                const int64_t u = (int64_t)s_unit[2 * first] + (int64_t)kv * ppages;
                x.prefix_count = segments(units, u, u + ppages - 1, &w0);
                x.prefix = record_entry(s_col[2 * first], rows, a.hkv, G, kv, w0) + (r - first) * G;
                x.step = kRecordCols;
                x.stream_step = -1;
            } else {
                const int chunks = chunks_of(rows), each = chunk_rows(rows, chunks), chunk = (r - first) / each, row0 = chunk * each;
                const int crows = min(each, rows - row0), cost = page_cost(rows, chunks, G), opens = job_start(cost);
                const int64_t u = s_cost[first] + ((int64_t)(kv * chunks + chunk) * (ppages + opens) + opens) * cost;
                const int n = segments(costs, u, u + (int64_t)(ppages - 1) * cost, &w0);
                const bool wide = chunk_wide(crows, G);
                x.prefix_count = wide ? n : 2 * n;
                x.prefix = run_entry(s_before[first], rows, a.hkv, G, kv, row0, w0) + (r - first - row0) * G;
                x.step = 4 * kTileRows;
                x.stream_step = wide ? 0 : crows * G;
            }
        }
        a.view.rows[i] = x;
    }
}

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int kv16_plan(const kv16_pool* pool, const kv_tables* tables, int32_t num_q_heads, int32_t batch,
                                 const int32_t* seq_ids, const int32_t* prefix_ids, void* workspace, int64_t workspace_bytes,
                                 int32_t* device_error, void* stream)
{
    if (int rc = kv16_check_heads(pool, num_q_heads, batch)) return rc;
    if (int rc = kv4_check_tables(tables)) return rc;
    if (!seq_ids && batch > tables->max_seqs)
        return kv4_fail(KVC_ERR_INVALID, "kv16_plan: more rows than requests, and no seq_ids");
    if (!kv4_aligned(seq_ids, 4) || !kv4_aligned(prefix_ids, 4) || !kv4_aligned(tables->lens, 4))
        return kv4_fail(KVC_ERR_INVALID, "kv16_plan: ids and lengths must be 4-byte aligned");
    if (!workspace || !kv4_aligned(workspace, 256)) return kv4_fail(KVC_ERR_INVALID, "kv16_plan: workspace must be 256-byte aligned");
    int sms = 0;
    if (int rc = kv16_sms(&sms)) return rc;
    StepPlanArgs a{};
    a.view = plan_view(workspace, batch, num_q_heads, pool->num_kv_heads, pool->head_dim, sms);
    if (workspace_bytes < a.view.bytes) return kv4_fail(KVC_ERR_INVALID, "kv16_plan: workspace must have kv16_workspace_bytes()");
    a.lens = tables->lens;
    a.seq_ids = seq_ids;
    a.prefix_ids = prefix_ids;
    a.max_seqs = tables->max_seqs;
    a.max_pages = tables->max_pages;
    a.batch = batch;
    a.hq = num_q_heads;
    a.hkv = pool->num_kv_heads;
    a.dim = pool->head_dim;
    a.grid = sms;
    a.err = device_error;
    static OncePerDevice once;
    if (cudaError_t e = once.set_attribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPlanRowBytes * kKv16MaxBatch);
        e != cudaSuccess)
        return kv4_launch_result(e);
    // Few rows: small blocks, whose scans and barriers are shorter, and more of them, so that a thread has no more than one start or
    // row of the merge (64 rows of 32 heads 5.2 us, in 16 blocks of 256 threads 7.8; 300 rows 11.1, with 1024 threads 16.5).
    const int threads = batch <= 64 ? 64 : batch <= 128 ? 128 : batch <= 256 ? 256 : kPlanMaxThreads, ctas = threads == 64 ? 128 : threads == 512 ? 16 : 64;
    return kv4_launch_result(kv4_launch(plan_kernel, dim3(ctas), threads, (size_t)kPlanRowBytes * batch, static_cast<cudaStream_t>(stream), a));
}
