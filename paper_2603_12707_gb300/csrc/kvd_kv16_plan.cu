// kv16_plan: the plan of a decode step over shared prefixes (kvd_kv16_plan.h),
// made by one CTA from the lengths on the device.  Runs of rows with one prefix come from a scan of maxima
// over their first rows, places in the two lines of work from scans of sums, each worker's start from a
// binary search.
#include "kvd_kv16_plan.h"

namespace kvd {
namespace {

constexpr int kPlanMaxThreads = 1024;

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
struct Max {
    int32_t v;
};
__device__ __forceinline__ Max operator+(const Max& a, const Max& b) { return {max(a.v, b.v)}; }
__device__ __forceinline__ Max shuffle_up(const Max& s, int n) { return {__shfl_up_sync(0xffffffffu, s.v, n)}; }

// Inclusive scan over the block's threads on top of `before`, which moves on by the total.
template <class S>
__device__ __forceinline__ S block_scan(S s, S* before, S* warp_sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll 1
    for (int n = 1; n < 32; n <<= 1) {
        const S o = shuffle_up(s, n);
        if (lane >= n) s = o + s;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    S start = *before;
#pragma unroll 1
    for (int i = 0; i < warps; ++i) {
        if (i == warp) s = start + s;
        start = start + warp_sums[i];
    }
    *before = start;
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

__global__ void __launch_bounds__(kPlanMaxThreads) plan_kernel(StepPlanArgs a)
{
    extern __shared__ int64_t shared[];
    int64_t* const s_cost = shared;                                   // [batch]
    int32_t* const s_unit = reinterpret_cast<int32_t*>(s_cost + a.batch);   // [2 * batch]
    int32_t* const s_pre = s_unit + 2 * a.batch;                      // [batch]: prefix, -1: none, of length 0 or refused
    int32_t* const s_rows = s_pre + a.batch;                          // [batch]: rows of the run that starts there
    __shared__ Sums sum_warps[kPlanMaxThreads / 32];
    __shared__ Max max_warps[kPlanMaxThreads / 32];
    const int tid = threadIdx.x, threads = blockDim.x, B = a.batch, G = a.hq / a.hkv;
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
    // Own lengths go through the records, prefixes through shared memory.
#pragma unroll 1
    for (int r = tid; r < B; r += threads) {
        const int req = a.seq_ids ? a.seq_ids[r] : r, pre = a.prefix_ids ? a.prefix_ids[r] : -1;
        bool bad = false;
        const int n = length(req, &bad), np = pre == -1 ? 0 : length(pre, &bad);
        any_bad |= bad;
        s_pre[r] = bad || np == 0 ? -1 : pre;
        Record own{};
        own.req = req;
        own.len = bad ? 0 : n;
        own.pages = bad ? 0 : pages_of(n);
        own.row0 = r;
        own.rows = 1;
        a.view.recs[2 * r + 1] = own;
    }
    if (any_bad) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
    __syncthreads();
    // Runs.
    Max before_max{-1};
#pragma unroll 1
    for (int r0 = 0; r0 < B; r0 += threads) {
        const int r = r0 + tid;
        const int pre = r < B ? s_pre[r] : -1;
        const bool starts = r < B && (r == 0 || s_pre[r - 1] != pre);
        const Max at = block_scan(Max{starts ? r : -1}, &before_max, max_warps);
        if (r < B) {
            a.view.row_run[r] = pre >= 0 ? at.v : -1;
            if (r + 1 == B || s_pre[r + 1] != pre) s_rows[at.v] = r + 1 - at.v;
        }
    }
    __syncthreads();
    // Places in the lines of work.
    Sums total{0, 0, 0, 0};
#pragma unroll 1
    for (int r0 = 0; r0 < B; r0 += threads) {
        const int r = r0 + tid;
        Sums mine{0, 0, 0, 0};
        Record own{}, small{};
        Run run{};
        if (r < B) {
            own = a.view.recs[2 * r + 1];
            const int pre = s_pre[r];
            if (pre >= 0 && (r == 0 || s_pre[r - 1] != pre)) {
                const int n = a.lens[pre], rows = s_rows[r], pages = pages_of(n);
                if (rows * G <= kRecordCols) {
                    small.req = pre;
                    small.len = n;
                    small.pages = pages;
                    small.row0 = r;
                    small.rows = rows;
                } else {
                    run.req = pre;
                    run.len = n;
                    run.pages = pages;
                    run.rows = rows;
                    const int pair = 2 * (kTileRows / G);
                    run.chunks = (rows + pair - 1) / pair;
                    // (nearly equal chunks: the last ones may be left without rows)
                    const int each = chunk_rows(rows, run.chunks);
                    run.chunks = (rows + each - 1) / each;
                    mine.cost = (int64_t)pages * a.hkv * run.chunks * page_cost(rows, run.chunks, G);
                    mine.rows = rows;
                }
            }
            mine.units = (int64_t)(small.pages + own.pages) * a.hkv;
            mine.cols = (small.rows + own.rows) * G;
        }
        const Sums at = block_scan(mine, &total, sum_warps);
        if (r < B) {
            const int64_t unit = at.units - mine.units;
            small.unit = (int32_t)unit;
            own.unit = (int32_t)(unit + (int64_t)small.pages * a.hkv);
            small.col = at.cols - mine.cols;
            own.col = small.col + small.rows * G;
            run.cost = at.cost - mine.cost;
            run.rows_before = at.rows - mine.rows;
            s_unit[2 * r] = small.unit;
            s_unit[2 * r + 1] = own.unit;
            s_cost[r] = run.cost;
            a.view.recs[2 * r] = small;
            a.view.recs[2 * r + 1] = own;
            a.view.runs[r] = run;
        }
    }
    const bool fits = total.units < (int64_t)1 << 31 && total.cost < (int64_t)1 << 40;
    // CTAs for large runs, the others for records: the cut at which the slower side is fastest.
    int ctas = 0;
    if (total.cost > 0) {
        const double c = (double)total.cost, u = (double)total.units * kRecordCost;
        ctas = a.grid;
        if (total.units > 0) {
            const int f = min(max((int)(a.grid * c / (c + u)), 1), a.grid - 1), g = min(f + 1, a.grid - 1);
            ctas = max(c / f, u / (a.grid - f)) <= max(c / g, u / (a.grid - g)) ? f : g;
        }
        const int64_t enough = total.cost / (2 * kWideCost);   // every worker has a page of each kind
        if (ctas > enough) ctas = (int)max(enough, (int64_t)1);
    }
    const int64_t slots = (int64_t)(a.grid - ctas) * kAttnWarps;
    const int64_t warps = min(slots, total.units);
    if (tid == 0) {
        if (!fits) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
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
        h.warps = (int)warps;
        h.units = total.units;
        h.cost = total.cost;
        *a.view.header = h;
    }
    __syncthreads();
    if (!fits) return;
#pragma unroll 1
    for (int w = tid; w < warps; w += threads) {
        const int32_t u = (int32_t)share_start(w, total.units, warps);
        const int i = last_at(s_unit, 2 * B, u);
        const int pages = a.view.recs[i].pages, off = u - s_unit[i];
        const int head = off / pages;
        a.view.warp_starts[w] = WarpStart{i, head, off - head * pages, 0};
    }
#pragma unroll 1
    for (int c = tid; c < ctas; c += threads) {
        const int64_t at = share_start(c, total.cost, ctas);
        int i = last_at(s_cost, B, at);
        const Run run = a.view.runs[i];
        const int w = page_cost(run.rows, run.chunks, G);
        const int64_t page = (at - run.cost + w - 1) / w;      // the first page that starts at or after the share
        const int64_t job = page / run.pages;
        a.view.cta_starts[c] = CtaStart{i, (int32_t)job, (int32_t)(page - job * run.pages), 0};   // (job: may be one past the run's last)
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
    constexpr int kRowBytes = 8 + 4 * 4;
    static OncePerDevice once;
    if (cudaError_t e = once.set_attribute(plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowBytes * kKv16MaxBatch);
        e != cudaSuccess)
        return kv4_launch_result(e);
    const int threads = batch <= 256 ? 256 : kPlanMaxThreads;   // (few rows: shorter scans and barriers)
    return kv4_launch_result(kv4_launch(plan_kernel, dim3(1), threads, (size_t)kRowBytes * batch, static_cast<cudaStream_t>(stream), a));
}
