// kv16_attention: decode attention of a batch whose rows share prefixes
// (kvdecode16.h), from the plan of kv16_plan (kvd_kv16_plan.h).
//
// For a row the softmax runs over its prefix's tokens and its own.  Both are
// cut into segments whose results (o = sum p v, m, l = sum p with p = 2^(s - m))
// a second launch merges.  One persistent CTA per SM works on one kind:
//
// * Prefixes of many rows: S = Q K^T with up to 256 query rows of a KV head against tiles of 128 tokens is a dense
//   contraction, done by tcgen05.  Two streams of four softmax warps each hold scores and outputs of 128
//   query rows in tensor memory (128 + head_dim columns); with more than 128 rows each has rows of
//   its own, else the streams take halves of a tile's tokens.  A warp loads tiles (TMA, a
//   ring of K and V tiles in shared memory), one thread issues the MMAs of both streams in turn, so that
//   one stream's products run while the other's scores are worked.  A thread owns a row: no exchange between
//   lanes.  Weights go back into tensor memory where their scores were, 16 bits each, as the
//   operand of P V.
// * A row's own tokens, and prefixes of few rows: a warp's worth of pages (16 tokens) at a
//   time, S^T = K q^T and O^T = V^T P^T on mma.sync with the query rows padded to 8 columns, each warp with a ring of its own.
//
// The reference m of a row moves only when a score exceeds it by more than 8 in log2 units (weights stay below 2^8).
// fp16 weights carry a factor 2^7 more, so that the small ones keep their bits.
#include <cudaTypedefs.h>
#include <math.h>

#include <mutex>

#include "kvd_kv16_plan.h"
#include "kvd_ptx.cuh"
#include "kvd_tcgen05.cuh"

namespace kvd {
namespace {

constexpr uint64_t kLimitNs = 1000000000ull;
constexpr int kThreads = 32 * kAttnWarps;
constexpr int kTilePages = 8;                      // of a tile of a large run: 128 tokens
constexpr int kLoadWarp = 8, kMmaWarp = 9;         // after two streams of four softmax warps

template <int D>
struct Geo {
    static constexpr int kBlocks = D / 64;                        // blocks of 64 columns (128 bytes)
    static constexpr int kBlockBytes = kTileRows * 128;           // of a tile of 128 rows
    static constexpr int kTileBytes = kBlocks * kBlockBytes;
    static constexpr int kSlots = D == 128 ? 5 : 9;               // tiles of K or V in the ring
    static constexpr int kRing = 2 * kTileBytes;                  // after two tiles of queries
    static constexpr int kPageBytes = kPageSize * D * 2;          // K, or V, of a page and KV head
    static constexpr int kStages = D == 128 ? 2 : 4;              // of a record warp's ring: K and V of a page each
    static constexpr int kWarpRing = kStages * 2 * kPageBytes;
    static constexpr int kData = kRing + kSlots * kTileBytes > kAttnWarps * kWarpRing ? kRing + kSlots * kTileBytes : kAttnWarps * kWarpRing;
    static constexpr int kSmem = kData + 1024;
};

template <class T>
struct Weights {   // weights in the pool's type: log2 of the factor that they carry
    static constexpr float kShift = 0.f;
};
template <>
struct Weights<Fp16> {
    static constexpr float kShift = 7.f;
};

struct AttnArgs {
    PlanView view;
    int32_t batch, hq, hkv, G, dim, grid;
    const uint16_t* q;
    int64_t q_stride;
    uint16_t* out;
    int64_t out_stride;
    float* lse;
    float scale_log2;
    const int32_t* table;
    int32_t max_seqs, max_pages;
    int64_t num_pages;
    int32_t* err;
};

struct Control {                     // in shared memory
    uint64_t full[16], empty[16];    // ring slots of large runs
    uint64_t scores[2], weights[2], output[2], queries, drained;   // by stream
    uint64_t stage[kAttnWarps][4];   // rings of record warps
    int32_t pages_known[8];          // by tile: bits of its pages that are there (a tile's scores are worked before the 5th after it is loaded)
    uint32_t tmem;
    int32_t gave_up;                 // a wait ran out: everybody leaves
};

__device__ __forceinline__ bool plan_fits(const PlanHeader& h, const AttnArgs& a)
{
    return h.magic == kPlanMagic && h.batch == a.batch && h.hq == a.hq && h.hkv == a.hkv && h.dim == a.dim && h.grid == a.grid &&
           h.max_seqs == a.max_seqs && h.max_pages == a.max_pages;
}

// All lanes of a warp wait; false for all where it took too long or others gave up.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, Control& c, int32_t* err)
{
    const uint32_t addr = smem_addr(bar);
    if (__all_sync(0xffffffffu, mbar_try_wait(addr, parity))) return true;
    const uint64_t t0 = global_timer_ns();
    while (true) {
        const bool ok = mbar_try_wait(addr, parity);
        const bool late = global_timer_ns() - t0 > kLimitNs || *reinterpret_cast<volatile int32_t*>(&c.gave_up);
        if (__all_sync(0xffffffffu, ok)) return true;
        if (__any_sync(0xffffffffu, late)) {
            *reinterpret_cast<volatile int32_t*>(&c.gave_up) = 1;
            if ((threadIdx.x & 31) == 0) kv4_error(err, KVC_DEVERR_WAIT_TIMEOUT);
            return false;
        }
    }
}

__device__ __forceinline__ bool thread_wait(uint64_t* bar, uint32_t parity, Control& c, int32_t* err)
{
    const uint32_t addr = smem_addr(bar);
    if (mbar_try_wait(addr, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    while (true) {
        if (mbar_try_wait(addr, parity)) return true;
        if (global_timer_ns() - t0 > kLimitNs || *reinterpret_cast<volatile int32_t*>(&c.gave_up)) {
            *reinterpret_cast<volatile int32_t*>(&c.gave_up) = 1;
            kv4_error(err, KVC_DEVERR_WAIT_TIMEOUT);
            return false;
        }
    }
}

__device__ __forceinline__ void arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// ------------------------------------------------------------ large runs, tcgen05
// A worker's segments: pages [page, stop) of a job.
struct Segment {
    int run, job, page, stop;
    Run r;
    int head, row0, rows;        // KV head, first batch row, batch rows
    bool wide;                   // each stream has rows of its own
    int rows0;                   // batch rows of stream 0 (wide), else of both
    __device__ __forceinline__ int tiles() const { return (stop - page + kTilePages - 1) / kTilePages; }
};

struct Segments {
    const AttnArgs& a;
    int run, job, page;
    int64_t end;                 // of this worker's share, in cost units
    __device__ __forceinline__ Segments(const AttnArgs& args, const PlanHeader& h, int worker) : a(args)
    {
        const CtaStart s = a.view.cta_starts[worker];
        run = s.run;
        job = s.job;
        page = s.page;
        end = share_start(worker + 1, h.cost, h.prefix_ctas);
    }
    __device__ __forceinline__ bool next(Segment& s)
    {
        while (run < a.batch) {
            s.r = a.view.runs[run];
            const int jobs = s.r.chunks * a.hkv;
            if (s.r.pages == 0 || job >= jobs) {
                run += s.r.pages == 0 ? 1 : s.r.rows;
                job = page = 0;
                continue;
            }
            const int w = page_cost(s.r.rows, s.r.chunks, a.G);
            const int64_t first = s.r.cost + (int64_t)job * s.r.pages * w, left = end - first;
            const int64_t stop = left <= 0 ? 0 : (left + w - 1) / w;
            s.run = run;
            s.job = job;
            s.page = page;
            s.stop = (int)(stop < s.r.pages ? stop : s.r.pages);
            if (s.stop <= page) return false;
            s.head = job / s.r.chunks;
            const int each = chunk_rows(s.r.rows, s.r.chunks), chunk = job - s.head * s.r.chunks;
            s.row0 = run + chunk * each;
            s.rows = min(each, s.r.rows - chunk * each);
            s.wide = chunk_wide(s.rows, a.G);
            s.rows0 = s.wide ? (s.rows + 1) / 2 : s.rows;
            ++job;
            page = 0;
            return true;
        }
        return false;
    }
};

// Pages of a tile, and of those the ones that a stream works on.
__device__ __forceinline__ int tile_pages(const Segment& s, int tile) { return min(kTilePages, s.stop - s.page - tile * kTilePages); }
__device__ __forceinline__ int stream_first(const Segment& s, int np, int stream) { return s.wide || stream == 0 ? 0 : (np + 1) / 2; }
__device__ __forceinline__ int stream_pages(const Segment& s, int np, int stream) { return s.wide ? np : stream == 0 ? (np + 1) / 2 : np / 2; }

template <int D>
__device__ __forceinline__ void load_tiles(const AttnArgs& a, const PlanHeader& h, Control& c, uint8_t* smem, const CUtensorMap* mk,
                                           const CUtensorMap* mv, int lane)
{
    using G = Geo<D>;
    Segments segs(a, h, blockIdx.x);
    Segment s;
    uint32_t n = 0, tile_no = 0;                          // tiles of K and V so far; of both
    const uint64_t policy = l2_policy_evict_first();
    const int p = lane % kTilePages, block = lane / kTilePages;
    bool fine = true;
    while (fine && segs.next(s)) {
        const int32_t* row = a.table + (int64_t)s.r.req * a.max_pages;
        const int tiles = s.tiles();
        int id = p < tile_pages(s, 0) ? row[s.page + p] : -1;
#pragma unroll 1
        for (int t = 0; t < tiles && fine; ++t, ++tile_no) {
            const int np = tile_pages(s, t);
            const int next = t + 1 < tiles && p < tile_pages(s, t + 1) ? row[s.page + (t + 1) * kTilePages + p] : -1;
            const bool known = p < np && id >= 0 && id < a.num_pages;
            const uint32_t mask = __ballot_sync(0xffffffffu, known) & 0xffu;
            if (mask != (1u << np) - 1u && lane == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
#pragma unroll 1
            for (int side = 0; side < 2; ++side, ++n) {   // K, V
                const int slot = n % G::kSlots;
                if (!(fine = warp_wait(&c.empty[slot], (n / G::kSlots & 1) ^ 1, c, a.err))) break;
                const uint32_t bar = smem_addr(&c.full[slot]);
                if (lane == 0) {
                    if (side == 0) c.pages_known[tile_no % 8] = (int32_t)mask;
                    mbar_arrive_expect_tx(bar, __popc(mask) * (uint32_t)G::kPageBytes);
                }
                __syncwarp();
                if (known && block < G::kBlocks)
                    tma_load_3d(smem_addr(smem + G::kRing + slot * G::kTileBytes + block * G::kBlockBytes + p * 2048), side ? mv : mk, 0,
                                (id * a.hkv + s.head) * kPageSize, block, bar, policy);
            }
            id = next;
        }
    }
    // Where others gave up: what is under way arrives before the CTA leaves.
    if (*reinterpret_cast<volatile int32_t*>(&c.gave_up))
        for (uint32_t i = n > G::kSlots ? n - G::kSlots : 0; i < n; ++i)
            mbar_wait_bounded(smem_addr(&c.full[i % G::kSlots]), i / G::kSlots & 1, kLimitNs);
}

template <int D, class T>
__device__ __forceinline__ void issue_products(const AttnArgs& a, const PlanHeader& h, Control& c, uint8_t* smem)
{
    using G = Geo<D>;
    constexpr bool kBf16 = std::is_same_v<T, Bf16>;
    Segments segs(a, h, blockIdx.x);
    Segment s;
    const uint32_t base = smem_addr(smem), tm = c.tmem;
    uint32_t n = 0, segment = 0, ready[2] = {0, 0};
    // K tiles of a stream against its queries.
    auto scores = [&](int stream, uint32_t slot, int np) {
        const int pages = stream_pages(s, np, stream);
        if (pages == 0) return;
        const uint32_t q = base + (s.wide ? stream * G::kTileBytes : 0);
        const uint32_t k = base + G::kRing + slot * G::kTileBytes + stream_first(s, np, stream) * 2048;
        const uint32_t idesc = mma_desc(kBf16, false, kTileRows, pages * kPageSize);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t off = (ks / 4) * G::kBlockBytes + (ks % 4) * 32;
            mma_ss(tm + stream * 128, smem_desc(q + off, 16, 1024), smem_desc(k + off, 16, 1024), idesc, ks > 0);
        }
    };
    // A stream's weights against V.
    auto outputs = [&](int stream, uint32_t slot, int np, bool add) {
        const int pages = stream_pages(s, np, stream);
        const uint32_t v = base + G::kRing + slot * G::kTileBytes + stream_first(s, np, stream) * 2048;
        const uint32_t idesc = mma_desc(kBf16, true, kTileRows, D);
#pragma unroll 1
        for (int kk = 0; kk < pages; ++kk)
            mma_ts(tm + 256 + stream * 128, tm + stream * 128 + kk * 8, smem_desc(v + kk * 2048, G::kBlockBytes, 1024), idesc, add || kk > 0);
    };
    while (segs.next(s)) {
        const int tiles = s.tiles();
        if (!thread_wait(&c.queries, segment & 1, c, a.err)) return;
        uint32_t slot = n % G::kSlots;
        if (!thread_wait(&c.full[slot], n / G::kSlots & 1, c, a.err)) return;
        tmem_fence_after();
        for (int st = 0; st < 2; ++st) {
            scores(st, slot, tile_pages(s, 0));
            mma_commit(smem_addr(&c.scores[st]));
            arrive(&c.scores[st]);       // (what the loading warp has said of the tile comes along)
        }
        mma_commit(smem_addr(&c.empty[slot]));
        ++n;
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
            const uint32_t vslot = n % G::kSlots, vpar = n / G::kSlots & 1;
            ++n;
            const uint32_t kslot = n % G::kSlots, kpar = n / G::kSlots & 1;
            const bool more = t + 1 < tiles;
            const int np = tile_pages(s, t), np2 = more ? tile_pages(s, t + 1) : 0;
            if (!thread_wait(&c.full[vslot], vpar, c, a.err)) return;
#pragma unroll 1
            for (int st = 0; st < 2; ++st) {
                if (!thread_wait(&c.weights[st], ready[st]++ & 1, c, a.err)) return;
                tmem_fence_after();
                outputs(st, vslot, np, t > 0);
                if (st == 1) mma_commit(smem_addr(&c.empty[vslot]));
                if (more) {
                    if (st == 0 && !thread_wait(&c.full[kslot], kpar, c, a.err)) return;
                    scores(st, kslot, np2);
                    mma_commit(smem_addr(&c.scores[st]));
                    arrive(&c.scores[st]);
                    if (st == 1) mma_commit(smem_addr(&c.empty[kslot]));
                } else {
                    mma_commit(smem_addr(&c.output[st]));
                }
            }
            if (more) ++n;
        }
        ++segment;
    }
}

// Bits of a tile's 128 tokens, from a stream's first page on, that take part.
__device__ __forceinline__ uint32_t token_bits(int word, int first_page, int pages, uint32_t known, int valid)
{
    // valid: tokens of the tile before the prefix's end
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int pg = 2 * word + i;
        if (pg < pages && (known >> (first_page + pg) & 1u)) {
            const int n = min(max(valid - (first_page + pg) * kPageSize, 0), kPageSize);
            m |= ((1u << n) - 1u) << (16 * i);
        }
    }
    return m;
}

template <int D, class T>
__device__ __forceinline__ void softmax_stream(const AttnArgs& a, const PlanHeader& h, Control& c, uint8_t* smem)
{
    using G = Geo<D>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, stream = warp >> 2, wq = warp & 3;
    const int my = wq * 32 + lane;                        // row of the stream's tile
    const uint32_t tm = c.tmem + ((uint32_t)wq << 21), ts = tm + stream * 128, to = tm + 256 + stream * 128;
    Segments segs(a, h, blockIdx.x);
    Segment s;
    uint32_t n = 0, segment = 0, tile_no = 0;
    const float sl = a.scale_log2;
    while (segs.next(s)) {
        // Queries: 16-byte chunks of up to 256 rows, in the tiles' swizzle.
        if (segment > 0 && !warp_wait(&c.drained, (segment - 1) & 1, c, a.err)) return;
        const int total = s.rows * a.G;
        for (int i = threadIdx.x; i < total * (D / 8); i += 256) {
            const int qr = i / (D / 8), ch = i % (D / 8), br = qr / a.G, g = qr - br * a.G;
            const int tile = br >= s.rows0, r = qr - tile * s.rows0 * a.G;
            const uint4 x = *reinterpret_cast<const uint4*>(a.q + (s.row0 + br) * a.q_stride + (int64_t)(s.head * a.G + g) * D + ch * 8);
            *reinterpret_cast<uint4*>(smem + tile * G::kTileBytes + (ch >> 3) * G::kBlockBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = x;
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) arrive(&c.queries);
        const int qrows = (s.wide ? (stream == 0 ? s.rows0 : s.rows - s.rows0) : s.rows) * a.G;
        const bool works = wq * 32 < qrows;               // (the others have no row of the tile)
        float ref = -INFINITY, l = 0.f;
        bool some = false;                                // products with V so far
        const int tiles = s.tiles();
#pragma unroll 1
        for (int t = 0; t < tiles; ++t, ++tile_no, n += 2) {
            const int np = tile_pages(s, t), pages = stream_pages(s, np, stream), first = stream_first(s, np, stream);
            const uint32_t vslot = (n + 1) % G::kSlots;
            if (!warp_wait(&c.scores[stream], tile_no & 1, c, a.err)) return;
            tmem_fence_after();
            const uint32_t known = (uint32_t)c.pages_known[tile_no % 8];
            const int valid = s.r.len - (s.page + t * kTilePages) * kPageSize;
            const bool whole = valid >= np * kPageSize && known == (1u << np) - 1u;
            if (works && pages > 0) {
                const int words = (pages + 1) / 2;
                const bool plain = whole && (pages & 1) == 0;
                float mx = -INFINITY;
#pragma unroll 1
                for (int w = 0; w < words; ++w) {
                    uint32_t x[32];
                    tmem_ld32(ts + 32 * w, x);
                    tmem_wait_ld();
                    if (plain) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) mx = fmaxf(mx, __uint_as_float(x[i]));
                    } else {
                        const uint32_t bits = token_bits(w, first, pages, known, valid);
#pragma unroll
                        for (int i = 0; i < 32; ++i) mx = bits >> i & 1u ? fmaxf(mx, __uint_as_float(x[i])) : mx;
                    }
                }
                mx *= sl;
                const float top = fmaxf(ref, mx);
                if (__any_sync(0xffffffffu, mx > ref + 8.f)) {
                    if (some) {
                        const float alpha = ref == top ? 1.f : ex2(ref - top);
                        l *= alpha;
#pragma unroll 1
                        for (int w = 0; w < D / 32; ++w) {
                            uint32_t x[32];
                            tmem_ld32(to + 32 * w, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * alpha);
                            tmem_st32(to + 32 * w, x);
                        }
                    }
                    ref = top;
                }
                const float sub = (ref == -INFINITY ? 0.f : ref) - Weights<T>::kShift;
                float sum = 0.f;
#pragma unroll 1
                for (int w = 0; w < words; ++w) {
                    uint32_t x[32], p[16];
                    tmem_ld32(ts + 32 * w, x);
                    tmem_wait_ld();
                    if (plain) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(ex2(fmaf(__uint_as_float(x[i]), sl, -sub)));
                    } else {
                        const uint32_t bits = token_bits(w, first, pages, known, valid);
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] = bits >> i & 1u ? __float_as_uint(ex2(fmaf(__uint_as_float(x[i]), sl, -sub))) : 0u;
                    }
                    float part = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float u = __uint_as_float(x[2 * i]), v = __uint_as_float(x[2 * i + 1]);
                        part += u + v;
                        p[i] = T::pack(u, v);
                    }
                    sum += part;
                    tmem_st16(ts + 16 * w, p);
                }
                l += sum;
                tmem_wait_st();
            }
            some |= pages > 0;
            if (!whole) {   // rows of V that hold anything: zero, or 0 * NaN would reach the sums
                if (!warp_wait(&c.full[vslot], (n + 1) / G::kSlots & 1, c, a.err)) return;
                for (int r = first * kPageSize + wq; r < (first + pages) * kPageSize; r += 4)
                    if (r >= valid || !(known >> (r / kPageSize) & 1u))
                        for (int b = 0; b < G::kBlocks; ++b)
                            *reinterpret_cast<uint32_t*>(smem + G::kRing + vslot * G::kTileBytes + b * G::kBlockBytes + r * 128 + lane * 4) = 0u;
                fence_proxy_async_smem();
            }
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) arrive(&c.weights[stream]);
        }
        if (!warp_wait(&c.output[stream], segment & 1, c, a.err)) return;
        tmem_fence_after();
        if (works) {
            // Rows of 32 columns through shared memory (this warp's 4 KB of the query tiles, which all products
            // have read by now), so that a row's columns are stored together.
            const int64_t entry = run_entry(s.r, a.hkv, a.G, s.head, s.row0 - s.run, blockIdx.x) +
                                  (int64_t)(stream == 0 ? 0 : (s.wide ? s.rows0 : s.rows) * a.G);
            uint8_t* const mine = smem + warp * 4096;
            if (my < qrows) a.view.run_ml[entry + my] = make_float2(some ? ref - Weights<T>::kShift : -INFINITY, some ? l : 0.f);
#pragma unroll 1
            for (int w = 0; w < D / 32; ++w) {
                uint32_t x[32];
                tmem_ld32(to + 32 * w, x);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<uint4*>(mine + lane * 128 + ((i ^ (lane & 7)) << 4)) =
                        some ? make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]) : make_uint4(0, 0, 0, 0);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 4 * i + (lane >> 3), ch = lane & 7;
                    const uint4 v = *reinterpret_cast<const uint4*>(mine + r * 128 + ((ch ^ (r & 7)) << 4));
                    if (wq * 32 + r < qrows) *reinterpret_cast<uint4*>(a.view.run_o + (entry + wq * 32 + r) * D + w * 32 + ch * 4) = v;
                }
                __syncwarp();
            }
        }
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) arrive(&c.drained);
        ++segment;
    }
}

// ----------------------------------------------------------- records, mma.sync
// Byte offset of 16-byte chunk ch of row r in a page's tile: blocks of [16 rows][64 columns], 128-byte swizzle.
__device__ __forceinline__ uint32_t page_at(int r, int ch) { return (uint32_t)((ch >> 3) * 2048 + r * 128 + (((ch & 7) ^ (r & 7)) << 4)); }

template <class T>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same_v<T, Bf16>) mma_bf16_16816(c, a0, a1, a2, a3, b0, b1);
    else mma_f16_16816(c, a0, a1, a2, a3, b0, b1);
}

// Walks a worker's pages in windows of up to 32 of one record, with the page ids of the next window under way.
struct Windows {
    const AttnArgs& a;
    int rec, head, page, left;      // of the window to be loaded next
    Record r;
    int32_t ids = -1, next_ids = -1;   // this lane's page of the current window, and of the next
    int n = 0, next_n = 0, at = 0;     // pages of them; the current page
    int cur_head = 0, next_head = 0;

    __device__ __forceinline__ Windows(const AttnArgs& args, const WarpStart& s, int count) : a(args)
    {
        rec = s.rec;
        head = s.head;
        page = s.page;
        left = count;
        r = a.view.recs[rec];
        fetch();
        shift();
    }
    __device__ __forceinline__ void fetch()
    {
        next_n = 0;
        if (left <= 0) return;
        while (page >= r.pages) {   // the next job with pages
            page = 0;
            if (r.pages > 0 && head + 1 < a.hkv) {
                ++head;
                break;
            }
            head = 0;
            r = a.view.recs[++rec];
        }
        next_n = min(min(32, r.pages - page), left);
        const int lane = threadIdx.x & 31;
        next_ids = lane < next_n ? a.table[(int64_t)r.req * a.max_pages + page + lane] : -1;
        next_head = head;
        page += next_n;
        left -= next_n;
    }
    __device__ __forceinline__ void shift()
    {
        ids = next_ids;
        n = next_n;
        cur_head = next_head;
        at = 0;
        fetch();
    }
    __device__ __forceinline__ bool done() const { return n == 0; }
    __device__ __forceinline__ int id() const { return __shfl_sync(0xffffffffu, ids, at); }
    __device__ __forceinline__ void step()
    {
        if (++at == n) shift();
    }
};

template <int D, class T>
__device__ __forceinline__ void work_records(const AttnArgs& a, const PlanHeader& h, Control& c, uint8_t* smem, const CUtensorMap* mk,
                                             const CUtensorMap* mv)
{
    using G = Geo<D>;
    constexpr int KS = D / 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ctas = a.grid - h.prefix_ctas;
    const int worker = warp * ctas + (int)blockIdx.x - h.prefix_ctas;   // (few workers: spread over the SMs)
    if (worker >= h.warps) return;
    const int64_t u0 = share_start(worker, h.units, h.warps);
    int left = (int)(share_start(worker + 1, h.units, h.warps) - u0);
    const WarpStart start = a.view.warp_starts[worker];
    uint8_t* const ring = smem + warp * G::kWarpRing;
    const uint64_t policy = l2_policy_evict_first();

    // The ring's side: a page's K and V by lanes of 64 columns each.
    Windows win(a, start, left);
    uint32_t skipped = 0, phase = 0;                 // bits by stage: a page that is not there; the barrier's parity
    int put = 0, staged = 0;
    auto load = [&] {
        if (win.done()) return;
        const int id = win.id();
        const bool known = id >= 0 && id < a.num_pages;
        const uint32_t bar = smem_addr(&c.stage[warp][put]);
        if (known) {
            skipped &= ~(1u << put);
            if (lane == 0) mbar_arrive_expect_tx(bar, 2 * G::kPageBytes);
            __syncwarp();
            if (lane < 2 * G::kBlocks) {
                const int side = lane / G::kBlocks, block = lane % G::kBlocks;
                tma_load_3d(smem_addr(ring + (put * 2 + side) * G::kPageBytes + block * 2048), side ? mv : mk, 0,
                            (id * a.hkv + win.cur_head) * kPageSize, block, bar, policy);
            }
        } else {
            skipped |= 1u << put;
            if (lane == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
        }
        put = put + 1 == G::kStages ? 0 : put + 1;
        ++staged;
        win.step();
    };
    for (int i = 0; i < G::kStages; ++i) load();

    int rec = start.rec, head = start.head, page = start.page, get = 0;
    bool fine = true;
    while (left > 0 && fine) {
        const Record r = a.view.recs[rec];
        const int stop = min(r.pages, page + left);
        // Queries as columns: B fragments, column lane / 4.
        const int cols = r.rows * a.G, col = lane >> 2;
        uint32_t qb[KS][2];
        {
            const int br = col / a.G, g = col - br * a.G;
            const uint16_t* row = a.q + (int64_t)(r.row0 + (col < cols ? br : 0)) * a.q_stride + (int64_t)(head * a.G + (col < cols ? g : 0)) * D;
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) {
                const uint32_t x = reinterpret_cast<const uint32_t*>(row)[4 * i + (lane & 3)];
                qb[i >> 1][i & 1] = col < cols ? x : 0u;
            }
        }
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[KS][4];
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
        left -= stop - page;
#pragma unroll 1
        for (; page < stop; ++page) {
            if (!(skipped >> get & 1u)) {
                if (!(fine = warp_wait(&c.stage[warp][get], phase >> get & 1u, c, a.err))) break;
                phase ^= 1u << get;
                const uint32_t sk = smem_addr(ring + get * 2 * G::kPageBytes), sv = sk + G::kPageBytes;
                const int valid = r.len - page * kPageSize;
                float acc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
                const int ar = (lane & 7) + ((lane >> 3) & 1) * 8;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    uint32_t a0, a1, a2, a3;
                    ldsm_x4(sk + page_at(ar, ks * 2 + (lane >> 4)), a0, a1, a2, a3);
                    mma_16816<T>(acc[ks & 1], a0, a1, a2, a3, qb[ks][0], qb[ks][1]);
                }
                float sc[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) sc[k] = (acc[0][k] + acc[1][k]) * a.scale_log2;
                // Lane: tokens lane / 4 and + 8, columns 2 (lane % 4) and + 1.
                const int t0 = lane >> 2;
                if (valid < kPageSize) {
                    if (t0 >= valid) sc[0] = sc[1] = -INFINITY;
                    if (t0 + 8 >= valid) sc[2] = sc[3] = -INFINITY;
                }
                const float x0 = fmaxf(sc[0], sc[2]), x1 = fmaxf(sc[1], sc[3]);
                if (__any_sync(0xffffffffu, x0 > m0 + 8.f || x1 > m1 + 8.f)) {
                    float y0 = x0, y1 = x1;
#pragma unroll
                    for (int k = 4; k < 32; k <<= 1) {
                        y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, k));
                        y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, k));
                    }
                    y0 = fmaxf(y0, m0);
                    y1 = fmaxf(y1, m1);
                    const float f0 = y0 == m0 ? 1.f : ex2(m0 - y0), f1 = y1 == m1 ? 1.f : ex2(m1 - y1);
                    m0 = y0;
                    m1 = y1;
                    l0 *= f0;
                    l1 *= f1;
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        o[i][0] *= f0;
                        o[i][1] *= f1;
                        o[i][2] *= f0;
                        o[i][3] *= f1;
                    }
                }
                const float s0 = (m0 == -INFINITY ? 0.f : m0) - Weights<T>::kShift, s1 = (m1 == -INFINITY ? 0.f : m1) - Weights<T>::kShift;
                const float p0 = ex2(sc[0] - s0), p1 = ex2(sc[1] - s1), p2 = ex2(sc[2] - s0), p3 = ex2(sc[3] - s1);
                l0 += p0 + p2;
                l1 += p1 + p3;
                // P^T as B fragments: [token][column] to [column][token].
                const uint32_t b0 = movmatrix_trans(T::pack(p0, p1)), b1 = movmatrix_trans(T::pack(p2, p3));
                // Tokens 2 (lane % 4) and + 1 of each 8 that take part: V may hold anything past the end.
                uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
                if (valid < kPageSize) {
                    const int t = 2 * (lane & 3);
                    keep0 = (t < valid ? 0xffffu : 0u) | (t + 1 < valid ? 0xffff0000u : 0u);
                    keep1 = (t + 8 < valid ? 0xffffu : 0u) | (t + 9 < valid ? 0xffff0000u : 0u);
                }
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    // A = V^T: rows d 16 i .., columns tokens; matrices (d 0-7, t 0-7), (d 8-15, t 0-7), (d 0-7, t 8-15), (d 8-15, t 8-15).
                    uint32_t a0, a1, a2, a3;
                    ldsm_x4_trans(sv + page_at((lane & 7) + (lane >> 4) * 8, i * 2 + ((lane >> 3) & 1)), a0, a1, a2, a3);
                    mma_16816<T>(o[i], a0 & keep0, a1 & keep0, a2 & keep1, a3 & keep1, b0, b1);
                }
                __syncwarp();
            }
            get = get + 1 == G::kStages ? 0 : get + 1;
            --staged;
            load();
        }
        if (!fine) break;
        // The segment's results: columns 2 (lane % 4) and + 1, elements 16 i + lane / 4 and + 8.
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, k);
            l1 += __shfl_xor_sync(0xffffffffu, l1, k);
        }
        const int64_t entry = record_entry(r, a.hkv, a.G, head, worker);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int cc = 2 * (lane & 3) + k;
            if (cc >= cols) continue;
            float* dst = a.view.rec_o + (entry + cc) * D + (lane >> 2);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                dst[16 * i] = o[i][k];
                dst[16 * i + 8] = o[i][k + 2];
            }
            if (lane < 4) a.view.rec_ml[entry + cc] = make_float2((k ? m1 : m0) - Weights<T>::kShift, k ? l1 : l0);
        }
        // The next job.
        if (left > 0) {
            page = 0;
            if (++head == a.hkv) {
                head = 0;
                do ++rec;
                while (a.view.recs[rec].pages == 0);
            }
        }
    }
    // Where a wait ran out: what is under way arrives before the CTA leaves.
    if (!fine)
        for (int i = 0; i < staged; ++i) {
            const int st = (get + i) % G::kStages;
            if (!(skipped >> st & 1u)) mbar_wait_bounded(smem_addr(&c.stage[warp][st]), phase >> st & 1u, kLimitNs);
        }
}

template <int D, class T>
__global__ void __launch_bounds__(kThreads, 1) attention_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                                                                const __grid_constant__ AttnArgs a)
{
    extern __shared__ uint8_t raw[];
    __shared__ Control c;
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid < 16) {
        mbar_init(smem_addr(&c.full[tid]), 1);
        mbar_init(smem_addr(&c.empty[tid]), 1);
    }
    if (tid < 2) {
        mbar_init(smem_addr(&c.scores[tid]), 2);
        mbar_init(smem_addr(&c.weights[tid]), 4);
        mbar_init(smem_addr(&c.output[tid]), 1);
    }
    if (tid == 2) mbar_init(smem_addr(&c.queries), 8);
    if (tid == 3) mbar_init(smem_addr(&c.drained), 8);
    if (tid == 4) c.gave_up = 0;
    if (lane < 4) mbar_init(smem_addr(&c.stage[warp][lane]), 1);
    if (tid == 0) {
        prefetch_tensormap(&mk);
        prefetch_tensormap(&mv);
    }
    fence_mbar_init();
    __syncthreads();
    griddep_wait();
    griddep_launch_dependents();
    const PlanHeader h = *a.view.header;
    if (!plan_fits(h, a)) {
        if (tid == 0 && blockIdx.x == 0) kv4_error(a.err, KVC_DEVERR_PLAN);
        return;
    }
    if ((int)blockIdx.x >= h.prefix_ctas) {
        work_records<D, T>(a, h, c, smem, &mk, &mv);
        return;
    }
    if (warp == kMmaWarp) tmem_alloc(smem_addr(&c.tmem), 512);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp < 8) {
        softmax_stream<D, T>(a, h, c, smem);
    } else if (warp == kLoadWarp) {
        load_tiles<D>(a, h, c, smem, &mk, &mv, lane);
    } else if (warp == kMmaWarp) {
        if (lane == 0) {
            issue_products<D, T>(a, h, c, smem);
            if (*reinterpret_cast<volatile int32_t*>(&c.gave_up)) {   // what is under way ends before the memory is freed
                mma_commit(smem_addr(&c.full[15]));
                mbar_wait_bounded(smem_addr(&c.full[15]), 0, kLimitNs);
            }
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == kMmaWarp) tmem_dealloc(c.tmem, 512);
}

// ---------------------------------------------------------------------- merge
// A warp per (row, query head): the partial results of the row's own segments, then its prefix's, in their order.
template <int D, class T>
__global__ void __launch_bounds__(128) merge_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr int N = D / 32;
    griddep_wait();
    griddep_launch_dependents();
    const PlanHeader h = *a.view.header;
    if (!plan_fits(h, a)) return;
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (unit >= (int64_t)a.batch * a.hq) return;
    const int row = (int)(unit / a.hq), head = (int)(unit - (int64_t)row * a.hq), kv = head / a.G, g = head - kv * a.G;

    // Segments: workers first .. first + count - 1 of up to two sources.
    struct Source {
        int64_t entry;     // of worker `first`
        int step, count;   // entries between workers; segments
    };
    Source src[2] = {{0, 0, 0}, {0, 0, 0}};
    int halves = 1;        // streams that share the rows of the prefix's job
    int64_t half_step = 0;
    auto record = [&](int i, int col, Source& s) {
        const Record r = a.view.recs[i];
        if (r.pages == 0) return;
        const int64_t u = (int64_t)r.unit + (int64_t)kv * r.pages;
        const int64_t w0 = share_of(u, h.units, h.warps), w1 = share_of(u + r.pages - 1, h.units, h.warps);
        s = {record_entry(r, a.hkv, a.G, kv, w0) + col, kRecordCols, (int)(w1 - w0) + 1};
    };
    record(2 * row + 1, g, src[0]);
    const int run = a.view.row_run[row];
    bool large = false;
    if (run >= 0) {
        const Run r = a.view.runs[run];
        large = r.pages > 0;
        if (large) {
            const int each = chunk_rows(r.rows, r.chunks), chunk = (row - run) / each, row0 = chunk * each;
            const int rows = min(each, r.rows - row0), w = page_cost(r.rows, r.chunks, a.G);
            const int64_t first = r.cost + (int64_t)(kv * r.chunks + chunk) * r.pages * w;
            const int64_t w0 = share_of(first, h.cost, h.prefix_ctas), w1 = share_of(first + (int64_t)(r.pages - 1) * w, h.cost, h.prefix_ctas);
            halves = chunk_wide(rows, a.G) ? 1 : 2;
            half_step = (int64_t)rows * a.G;
            src[1] = {run_entry(r, a.hkv, a.G, kv, row0, w0) + (row - run - row0) * a.G + g, 4 * kTileRows, (int)(w1 - w0 + 1) * halves};
        } else {
            record(2 * run, (row - run) * a.G + g, src[1]);
        }
    }
    float m = -INFINITY, l = 0.f, o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
    for (int k = 0; k < 2; ++k) {
        const bool of_run = k == 1 && large;
        const float2* ml = of_run ? a.view.run_ml : a.view.rec_ml;
        const float* po = of_run ? a.view.run_o : a.view.rec_o;
        for (int s0 = 0; s0 < src[k].count; s0 += 32) {
            const int s = s0 + lane, n = min(32, src[k].count - s0), by = of_run ? halves : 1;
            const int64_t e = src[k].entry + (int64_t)(s / by) * src[k].step + (s % by) * half_step;
            const float2 x = s < src[k].count ? ml[e] : make_float2(-INFINITY, 0.f);
            float top = x.y == 0.f ? -INFINITY : x.x;   // (a segment without tokens has no part)
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            top = fmaxf(top, m);
            const float old = m == top ? 1.f : ex2(m - top), mine = x.y == 0.f ? 0.f : x.x == top ? 1.f : ex2(x.x - top);
            float sum = x.y * mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            m = top;
            l = l * old + sum;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] *= old;
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const float wj = __shfl_sync(0xffffffffu, mine, j);
                const int64_t ej = __shfl_sync(0xffffffffu, e, j);
                const float* p = po + ej * D + lane * N;
                if constexpr (N == 4) {
                    const float4 v = *reinterpret_cast<const float4*>(p);
                    o[0] += wj * v.x;
                    o[1] += wj * v.y;
                    o[2] += wj * v.z;
                    o[3] += wj * v.w;
                } else {
                    const float2 v = *reinterpret_cast<const float2*>(p);
                    o[0] += wj * v.x;
                    o[1] += wj * v.y;
                }
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t* const dst = a.out + (int64_t)row * a.out_stride + (int64_t)head * D + lane * N;
    if constexpr (N == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv));
    else *reinterpret_cast<uint32_t*>(dst) = T::pack(o[0] * inv, o[1] * inv);
    if (a.lse && lane == 0) a.lse[(int64_t)row * a.hq + head] = l == 0.f ? -INFINITY : m * 0.693147180559945309f + logf(l);
}

PFN_cuTensorMapEncodeTiled_v12000 encoder()
{
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    });
    return fn;
}

// A pool's side as rows of head_dim elements, in boxes of 16 rows (a page's of one KV head) x 64 columns.
CUresult encode_pages(PFN_cuTensorMapEncodeTiled_v12000 encode, CUtensorMap* map, const kv16_pool& p, void* data)
{
    const cuuint64_t dims[3] = {64, (cuuint64_t)(p.num_pages * p.num_kv_heads * kPageSize), (cuuint64_t)(p.head_dim / 64)};
    const cuuint64_t strides[2] = {(cuuint64_t)p.head_dim * 2, 128};
    const cuuint32_t box[3] = {64, kPageSize, 1}, steps[3] = {1, 1, 1};
    return encode(map, p.dtype == KVC_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, data, dims, strides,
                  box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

template <int D, class T>
int launch_attention(const CUtensorMap& mk, const CUtensorMap& mv, const AttnArgs& a, cudaStream_t st)
{
    static OncePerDevice once;
    if (cudaError_t e = once.set_attribute(attention_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo<D>::kSmem); e != cudaSuccess)
        return kv4_launch_result(e);
    if (cudaError_t e = kv4_launch(attention_kernel<D, T>, dim3((unsigned)a.grid), kThreads, Geo<D>::kSmem, st, mk, mv, a); e != cudaSuccess)
        return kv4_launch_result(e);
    const int64_t units = (int64_t)a.batch * a.hq;
    return kv4_launch_result(kv4_launch(merge_kernel<D, T>, dim3((unsigned)((units + 3) / 4)), 128, 0, st, a));
}

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int64_t kv16_workspace_bytes(const kv16_pool* pool, int32_t num_q_heads, int32_t max_batch)
{
    if (int rc = kv16_check_heads(pool, num_q_heads, max_batch)) return rc;
    int sms = 0;
    if (int rc = kv16_sms(&sms)) return rc;
    return plan_view(nullptr, max_batch, num_q_heads, pool->num_kv_heads, pool->head_dim, sms).bytes;
}

extern "C" KVC_API int kv16_attention(const kv16_pool* pool, const kv_tables* tables, int32_t batch, int32_t num_q_heads,
                                      const void* q, int64_t q_stride, void* out, int64_t out_stride, float* lse,
                                      float softmax_scale, void* workspace, int64_t workspace_bytes, int32_t* device_error,
                                      void* stream)
{
    if (int rc = kv16_check_heads(pool, num_q_heads, batch)) return rc;
    if (int rc = kv16_check_pool(pool, true)) return rc;
    if (int rc = kv4_check_tables(tables)) return rc;
    if (!kv4_aligned(tables->block_table, 4)) return kv4_fail(KVC_ERR_INVALID, "kv16_attention: block_table must be 4-byte aligned");
    const int64_t width = (int64_t)num_q_heads * pool->head_dim;
    if (!kv16_rows_ok(q, q_stride, batch, 0, false) || !kv16_rows_ok(out, out_stride, batch, width, true))
        return kv4_fail(KVC_ERR_INVALID, "kv16_attention: q and out must be 16-byte aligned, their strides multiples of 8, out's rows apart");
    if (!kv4_aligned(lse, 4)) return kv4_fail(KVC_ERR_INVALID, "kv16_attention: lse must be 4-byte aligned");
    if (!(softmax_scale < 0x1p100f)) return kv4_fail(KVC_ERR_INVALID, "kv16_attention: softmax_scale must be below 2^100");
    if (!workspace || !kv4_aligned(workspace, 256)) return kv4_fail(KVC_ERR_INVALID, "kv16_attention: workspace must be 256-byte aligned");
    int sms = 0;
    if (int rc = kv16_sms(&sms)) return rc;
    AttnArgs a{};
    a.view = plan_view(workspace, batch, num_q_heads, pool->num_kv_heads, pool->head_dim, sms);
    if (workspace_bytes < a.view.bytes) return kv4_fail(KVC_ERR_INVALID, "kv16_attention: workspace must have kv16_workspace_bytes()");
    a.batch = batch;
    a.hq = num_q_heads;
    a.hkv = pool->num_kv_heads;
    a.G = num_q_heads / pool->num_kv_heads;
    a.dim = pool->head_dim;
    a.grid = sms;
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.out = static_cast<uint16_t*>(out);
    a.out_stride = out_stride;
    a.lse = lse;
    a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf((float)pool->head_dim)) * 1.4426950408889634f;
    a.table = tables->block_table;
    a.max_seqs = tables->max_seqs;
    a.max_pages = tables->max_pages;
    a.num_pages = pool->num_pages;
    a.err = device_error;
    const auto encode = encoder();
    if (!encode) return kv4_fail(KVC_ERR_CUDA, "kv16_attention: cuTensorMapEncodeTiled unavailable");
    CUtensorMap mk, mv;
    if (encode_pages(encode, &mk, *pool, pool->k) != CUDA_SUCCESS || encode_pages(encode, &mv, *pool, pool->v) != CUDA_SUCCESS)
        return kv4_fail(KVC_ERR_INVALID, "kv16_attention: cuTensorMapEncodeTiled rejected the pool");
    cudaStream_t const st = static_cast<cudaStream_t>(stream);
    if (pool->dtype == KVC_DTYPE_BF16)
        return pool->head_dim == 64 ? launch_attention<64, Bf16>(mk, mv, a, st) : launch_attention<128, Bf16>(mk, mv, a, st);
    return pool->head_dim == 64 ? launch_attention<64, Fp16>(mk, mv, a, st) : launch_attention<128, Fp16>(mk, mv, a, st);
}
