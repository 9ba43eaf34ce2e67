// The plan of a decode step over shared prefixes: what kv16_plan writes into
// the workspace and the kernels of kv16_attention read.  Not part of the ABI.
//
// Work comes in two kinds.  A *large run* is a run of rows that share a prefix
// and are more than 8 query rows of a KV head: its job is (run, KV head, chunk of
// at most 2 x 128 query rows) over the prefix's pages, done by whole CTAs on tcgen05.  Everything else
// is a *record*: a row's own tokens, or the prefix of a run of up to 8 query
// rows; its job is (record, KV head), done by single warps on mma.sync.
// Jobs of a kind follow one another in one line of cost units (records: pages)
// that is cut into equal shares, one for each worker; where worker i's share
// starts is i * total / workers, so who did what follows from a few sums.
#pragma once

#include <stdint.h>

#include "kvd_kv16.h"

namespace kvd {

constexpr int kAttnWarps = 12;          // of a CTA that work on records
constexpr int kRecordCols = 8;          // query rows of a record's job at most
constexpr int kTileRows = 128;          // query rows of one of a CTA's two streams
constexpr int kTilePages = 8;           // of a tile of a large run: 128 tokens
constexpr uint32_t kPlanMagic = 0x16a77e41u;
constexpr uint32_t kPlanGaveUp = 0x16a77e42u;   // of a plan by which attention gave up a wait: it serves no call any more, and outputs become NaN

// Cost of a page of a large run's job, with both streams on rows of their own or taking turns, and what opening and
// closing a job costs beside, in such pages; a record's page.  (In units of some 20 cycles of an SM; the minima are flat: with records at
// twice this, 64 rows of 32 heads on 701 tokens take 82.7 us a layer instead of 76.5; with 60 pages for opening a narrow job,
// 16 rows of 32 heads on 1000 tokens 14.3 instead of 13.2.)
__host__ __device__ inline int record_cost(int dim) { return dim / 16; }
constexpr int kWideCost = 24, kNarrowCost = 12, kWideStart = 20, kNarrowStart = 30;
// Shares are not made smaller than this (pages): every segment is one more result to merge.  (Records, a layer with 4, 2 and 1: one row of 16
// tokens, 28/4 heads, 9.7, 6.9 and 5.8 us; four of 1369 9.4, 9.45 and 11.0.  Runs with 4, 8 and 12: four rows on 1369 tokens 9.5, 9.6 and 10.9.)
constexpr int kLeastRunPages = 8, kLeastRecordPages = 2;

// `total` units cut into n shares; worker w's starts at w * total / n, as far as 20 bits after the point go (rounded up, so
// that the last one ends at the total).
struct Shares {
    int64_t each;       // in 2^-20 units
    float inverse;      // workers a unit
    int32_t n;
    __host__ __device__ int64_t start(int w) const { return w * each >> 20; }
    // The worker whose share holds unit u: an estimate that is one off at most, mended.
    __host__ __device__ int worker(int64_t u) const
    {
        int w = (int)((float)u * inverse);
        w = w < n - 1 ? w : n - 1;
        w -= w > 0 && start(w) > u;
        w += w + 1 < n && start(w + 1) <= u;
        return w;
    }
};
__host__ __device__ inline Shares make_shares(int64_t total, int n)   // total < 2^40, n < 2^12
{
    if (n == 0 || total == 0) return {0, 0.f, 0};
    // total * 2^20 / n in steps of 32 bits (a division of 64 takes the plan a microsecond)
    const uint32_t d = (uint32_t)n, high = (uint32_t)(total >> 16), q1 = high / d;
    const uint32_t low = (high - q1 * d) << 16 | (uint32_t)(total & 0xffff), q2 = low / d, rest = low - q2 * d;
    return {((((int64_t)q1 << 16) + q2) << 20) + ((rest << 20) + d - 1) / d, (float)n / (float)total, n};
}

struct PlanHeader {
    uint32_t magic;
    int32_t batch, hq, hkv, dim, grid, max_seqs, max_pages;   // what it was made for
    int32_t prefix_ctas;        // CTAs 0 .. are the workers of large runs
    int32_t pad;
    Shares units;               // pages x KV heads of all records
    Shares cost;                // of all large runs
};

struct Record {
    int32_t req, len, pages;    // pages 0: no work
    int32_t row0, rows;
    int32_t unit;               // first of its units
    int32_t col;                // query rows of one KV head in the records before it
    int32_t pad;
};

struct Run {                    // by its first row; pages 0 in the other rows
    int32_t req, len, pages, rows;
    int64_t cost;               // first of its cost units
    int32_t rows_before;        // in large runs before it
    int32_t chunks;             // row chunks of a KV head
};

// A worker's part of a large run's job.
struct Segment {
    int32_t pages;               // 0: no more segments
    int32_t valid;               // tokens from its first page to the prefix's end
    int32_t wide;                // the streams have rows of their own (else they take turns at the tiles)
    int32_t head, row0, rows;    // KV head, first batch row, batch rows
    int32_t rows0;               // batch rows of stream 0's tile
    int32_t first;               // its first page
    int64_t entry;               // of its results
    __host__ __device__ int tiles() const { return (pages + kTilePages - 1) / kTilePages; }
    __host__ __device__ int tile_pages(int t) const
    {
        const int left = pages - t * kTilePages;
        return left < kTilePages ? left : kTilePages;
    }
};

struct WarpStart {              // by CTA and warp: what a worker of records does
    int32_t worker;
    int32_t rec, head, page, count;   // where it starts; pages (0: it has none)
    Record r;
    int32_t pad[3];
};

struct CtaStart {               // where a worker of large runs starts, and the end of its share
    int32_t run, job;           // the job after the first segment
    int64_t end;
    Run r;
    Segment s;                  // the first segment
};

// What the merge has to know of a row and KV head: the segments of its own tokens' job and of its prefix's, and where the results
// of their first query head lie.
struct RowSources {
    int64_t own, prefix;        // first entries
    int32_t own_count, prefix_count;   // segments; of the prefix, both streams' where they share rows
    int32_t step;               // entries from one of the prefix's segments to the next
    int32_t stream_step;        // to the second stream's; 0: there is none.  -1: the prefix is a record
};

struct PlanView {
    PlanHeader* header;
    Record* recs;               // [2 * batch]: 2 r the small run that starts in row r, 2 r + 1 row r's own tokens
    Run* runs;                  // [batch]
    RowSources* rows;           // [batch][hkv]
    WarpStart* warp_starts;     // [grid * kAttnWarps]
    CtaStart* cta_starts;       // [grid]
    float* rec_o;               // partial results of records: [entries][dim], and (m, l)
    float2* rec_ml;
    float* run_o;               // of large runs
    float2* run_ml;
    int64_t bytes;
};

__host__ __device__ inline int64_t plan_round(int64_t x) { return (x + 255) & ~(int64_t)255; }

// Layout of the workspace; the same for all lengths.
__host__ __device__ inline PlanView plan_view(void* base, int batch, int hq, int hkv, int dim, int grid)
{
    PlanView v;
    char* const p = static_cast<char*>(base);
    int64_t at = 0;
    auto take = [&](int64_t n) {
        char* const q = p + at;
        at += plan_round(n);
        return q;
    };
    v.header = reinterpret_cast<PlanHeader*>(take(sizeof(PlanHeader)));
    v.recs = reinterpret_cast<Record*>(take((int64_t)sizeof(Record) * 2 * batch));
    v.runs = reinterpret_cast<Run*>(take((int64_t)sizeof(Run) * batch));
    v.rows = reinterpret_cast<RowSources*>(take((int64_t)sizeof(RowSources) * batch * hkv));
    v.warp_starts = reinterpret_cast<WarpStart*>(take((int64_t)sizeof(WarpStart) * grid * kAttnWarps));
    v.cta_starts = reinterpret_cast<CtaStart*>(take((int64_t)sizeof(CtaStart) * grid));
    // Entries of a record's segment: its query rows; segments are jobs and cuts between workers.
    const int64_t rec_entries = (int64_t)2 * batch * hq + (int64_t)kRecordCols * grid * kAttnWarps;
    // Of a large run's segment: its query rows, for both streams where they share them.
    const int64_t run_entries = (int64_t)2 * batch * hq + (int64_t)4 * kTileRows * grid;
    v.rec_ml = reinterpret_cast<float2*>(take(rec_entries * 8));
    v.run_ml = reinterpret_cast<float2*>(take(run_entries * 8));
    v.rec_o = reinterpret_cast<float*>(take(rec_entries * 4 * dim));
    v.run_o = reinterpret_cast<float*>(take(run_entries * 4 * dim));
    v.bytes = at;
    return v;
}

// x / d for x >= 0 and a quotient below 2^22.
__host__ __device__ inline int64_t divide(int64_t x, int32_t d)
{
    int64_t q = (int64_t)((float)x / (float)d);
    while (q * d > x) --q;
    while ((q + 1) * d <= x) ++q;
    return q;
}

// Chunks of a large run's rows: nearly equal, of up to 2 * (128 / G) batch rows.
__host__ __device__ inline int chunk_rows(int rows, int chunks) { return (rows + chunks - 1) / chunks; }
__host__ __device__ inline bool chunk_wide(int crows, int G) { return crows * G > kTileRows; }
__host__ __device__ inline int page_cost(int rows, int chunks, int G)
{
    return chunk_wide(chunk_rows(rows, chunks), G) ? kWideCost : kNarrowCost;
}
__host__ __device__ inline int job_start(int cost) { return cost == kWideCost ? kWideStart : kNarrowStart; }
// x / cost rounded up, x >= 0, by either cost of a page.
__host__ __device__ inline int64_t pages_at(int64_t x, int cost) { return cost == kWideCost ? (x + kWideCost - 1) / kWideCost : (x + kNarrowCost - 1) / kNarrowCost; }

// First entries of partial results.
__host__ __device__ inline int64_t record_entry(int col, int rows, int hkv, int G, int head, int worker)
{
    return (int64_t)col * hkv + (int64_t)head * rows * G + kRecordCols * worker;
}
__host__ __device__ inline int64_t run_entry(int rows_before, int rows, int hkv, int G, int head, int row_in_run, int worker)
{
    return (int64_t)2 * G * ((int64_t)rows_before * hkv + (int64_t)head * rows + row_in_run) + 4 * kTileRows * worker;
}

// The segment of a worker whose share ends at `end`: job `job` of the run from page `page` on.  pages 0: the share ends
// before it.
__host__ __device__ inline Segment make_segment(const Run& r, int run, int job, int page, int64_t end, int hkv, int G, int worker)
{
    Segment s{};
    const int each = chunk_rows(r.rows, r.chunks), cost = chunk_wide(each, G) ? kWideCost : kNarrowCost, opens = job_start(cost);
    const int64_t left = end - (r.cost + (int64_t)job * (r.pages + opens) * cost);
    if (left <= 0) return s;
    int64_t stop = pages_at(left, cost) - opens;
    if (stop > r.pages) stop = r.pages;
    if (stop <= page) return s;
    s.head = job / r.chunks;
    const int first = (job - s.head * r.chunks) * each;
    s.pages = (int)stop - page;
    s.valid = r.len - page * kPageSize;
    s.row0 = run + first;
    s.rows = each < r.rows - first ? each : r.rows - first;
    s.wide = chunk_wide(s.rows, G);
    s.rows0 = s.wide ? (s.rows + 1) / 2 : s.rows;
    s.first = page;
    s.entry = run_entry(r.rows_before, r.rows, hkv, G, s.head, first, worker);
    return s;
}

}  // namespace kvd
