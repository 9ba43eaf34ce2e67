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

constexpr int kAttnWarps = 12;          // of a CTA; the workers of records
constexpr int kRecordCols = 8;          // query rows of a record's job at most
constexpr int kTileRows = 128;          // query rows of one of a CTA's two streams
constexpr uint32_t kPlanMagic = 0x16a77e41u;

struct PlanHeader {
    uint32_t magic;
    int32_t batch, hq, hkv, dim, grid, max_seqs, max_pages;   // what it was made for
    int32_t prefix_ctas;        // CTAs 0 .. are the workers of large runs
    int32_t warps;              // workers of records
    int64_t units;              // pages x KV heads of all records
    int64_t cost;               // of all large runs
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

struct WarpStart {              // where a worker of records starts
    int32_t rec, head, page, pad;
};

struct CtaStart {               // where a worker of large runs starts
    int32_t run, job, page, pad;
};

// Cost of a page of a large run's job: with both streams on rows of their own, or on halves of a tile's tokens.
// A record's page costs kRecordCost.
constexpr int kRecordCost = 16, kWideCost = 13, kNarrowCost = 7;

struct PlanView {
    PlanHeader* header;
    Record* recs;               // [2 * batch]: 2 r the small run that starts in row r, 2 r + 1 row r's own tokens
    Run* runs;                  // [batch]
    int32_t* row_run;           // [batch]: first row of the run that row r is in, -1: none
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
    v.row_run = reinterpret_cast<int32_t*>(take((int64_t)4 * batch));
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

// Start of worker w's share of `total` units among n workers, and the worker whose share holds unit u.
__host__ __device__ inline int64_t share_start(int64_t w, int64_t total, int64_t n) { return w * total / n; }
__host__ __device__ inline int64_t share_of(int64_t u, int64_t total, int64_t n) { return ((u + 1) * n - 1) / total; }

// Chunks of a large run's rows: nearly equal, of up to 2 * (128 / G) batch rows.
__host__ __device__ inline int chunk_rows(int rows, int chunks) { return (rows + chunks - 1) / chunks; }
__host__ __device__ inline bool chunk_wide(int crows, int G) { return crows * G > kTileRows; }
__host__ __device__ inline int page_cost(int rows, int chunks, int G)
{
    return chunk_wide(chunk_rows(rows, chunks), G) ? kWideCost : kNarrowCost;
}

// First entries of partial results.
__host__ __device__ inline int64_t record_entry(const Record& r, int hkv, int G, int head, int64_t worker)
{
    return (int64_t)r.col * hkv + (int64_t)head * r.rows * G + kRecordCols * worker;
}
__host__ __device__ inline int64_t run_entry(const Run& r, int hkv, int G, int head, int row_in_run, int64_t worker)
{
    return (int64_t)2 * G * ((int64_t)r.rows_before * hkv + (int64_t)head * r.rows + row_in_run) + 4 * kTileRows * worker;
}

}  // namespace kvd
