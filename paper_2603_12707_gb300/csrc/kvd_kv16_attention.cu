// kv16_attention: decode attention of a batch whose rows share prefixes
// (kvdecode16.h), from the plan of kv16_plan (kvd_kv16_plan.h).
//
// For a row the softmax runs over its prefix's tokens and its own.  Both are
// cut into segments whose results (o = sum p v, m, l = sum p with p = 2^(s - m))
// a second launch merges.  One persistent CTA per SM works on one kind:
//
// * Prefixes of many rows: S = Q K^T with up to 256 query rows of a KV head against tiles of 128 tokens is a dense
//   contraction, done by tcgen05.  Two streams of four softmax warps each have scores, weights and sums of 128
//   query rows in tensor memory; with more than 128 rows each has rows of its own ("wide"), else the streams take turns at the
//   tiles.  A thread owns a row: no exchange between lanes.  A ninth warp loads tiles (TMA, a ring of K and V tiles in shared
//   memory) and tells the others of segments, one more for each stream issues its products.  Weights go back into tensor memory, 16 bits
//   each, as the operand of P V, half a tile at a time, so that the first half meets V while the second is worked.
//   A tile of 256 rows takes 3000 cycles, of which the tensor pipe is busy 2050.  Bound by the columns that both streams' scores
//   pass through by turns: 512 cycles of products, 490 until four warps have them in registers, some 360 for the two hand-overs, twice
//   a tile (half of the exponentials, no search for the largest score or no rounding change its time by 2 % at most).  One prefix of
//   131009 tokens, 96 rows of 28/4 heads: 151 us a layer, 1.19 PFLOP/s.
// * A row's own tokens, and prefixes of up to 8 query rows: a warp takes a page (16 tokens) at a
//   time, S^T = K q^T and O^T = V^T P^T on mma.sync with the query rows padded to 8 columns, each warp with a ring of its own.
//   Bound by reading K and V: 64 rows of 32/32 heads and 640 to 1344 tokens 155 us a layer, 6.7 TB/s.
//
// The reference m of a row moves only when a score exceeds it by more than 8 in log2 units (weights stay at or below 2^8).
// fp16 weights carry a factor 2^7 more, so that the small ones keep their bits; m does not, since sums and denominators both do.
// Differences to the reference are taken before anything is added to them: far out, where the numbers of 32 bits are 2 apart and more,
// m - 7 and m + 8 would be rounded to others, and weights with them past 2^16.
#include <cudaTypedefs.h>
#include <math.h>

#include <mutex>

#include "kvd_kv16_plan.h"
#include "kvd_ptx.cuh"
#include "kvd_tcgen05.cuh"

namespace kvd {
namespace {

constexpr uint64_t kLimitNs = 1000000000ull;       // of waits for copies before leaving
constexpr long long kLimitCycles = 2000000000ll;   // of all others: a second
constexpr int kSoftmaxWarps = 8;                   // two streams of four
constexpr int kThreads = 32 * (kSoftmaxWarps + 4);
static_assert(kThreads == 32 * kAttnWarps);
// Registers of a thread at launch, and then by what its warp does.  (A row's 128 scores have to stay in registers: with 168 for
// all some spill, and the tile above takes 4600 cycles.)
constexpr int kRegisters = 168, kSoftmaxRegisters = 208, kOtherRegisters = 88;
constexpr int kMovedRegisters = kSoftmaxWarps * kSoftmaxRegisters + 4 * kOtherRegisters;   // of a lane of each warp
static_assert(kMovedRegisters <= (kSoftmaxWarps + 4) * kRegisters);
constexpr int kLoadWarp = kSoftmaxWarps, kMmaWarp = kSoftmaxWarps + 1;
constexpr int kOut = 256;                          // first column of the sums in tensor memory

template <int D>
struct Geo {
    static constexpr int kBlocks = D / 64;                        // blocks of 64 columns (128 bytes)
    static constexpr int kQueryBlock = kTileRows * 128;           // bytes of a block of a tile of queries
    static constexpr int kQueryTile = kBlocks * kQueryBlock;
    static constexpr int kBlockBytes = kTilePages * kPageSize * 128;   // of a block of a tile of K or V
    static constexpr int kTileBytes = kBlocks * kBlockBytes;
    static constexpr int kSlots = D == 128 ? 5 : 9;               // tiles of K or V in the ring
    static constexpr int kRing = 2 * kQueryTile;                  // after two tiles of queries
    static constexpr int kPageBytes = kPageSize * D * 2;          // K, or V, of a page and KV head
    static constexpr int kStages = D == 128 ? 2 : 4;              // of a record warp's ring: K and V of a page each
    static constexpr int kWarpRing = kStages * 2 * kPageBytes;
    static constexpr int kData = kRing + kSlots * kTileBytes > kAttnWarps * kWarpRing ? kRing + kSlots * kTileBytes : kAttnWarps * kWarpRing;
};

template <class T>
struct Weights {   // weights in the pool's type: log2 of the factor that they carry; and the type's largest number
    static constexpr float kShift = 0.f, kMost = 0x1.fep127f;
};
template <>
struct Weights<Fp16> {
    static constexpr float kShift = 7.f, kMost = 65504.f;
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

constexpr float kFar = 0x1p20f;      // references from here on, in log2 units: half a unit in their last place is 2^-4 and more

constexpr int kSegments = 8;         // told ahead: the ring has room for K and V of less than five tiles

struct Control {                     // in shared memory
    // The ring's slots.  Copies end in any order, and a stream that takes turns passes over slots of the other's tiles: the tile
    // before may still be on its way to a slot when this stream comes to wait for the next.  So a slot has two barriers, for every
    // other tile; the tile two before has been used (the loading warp found it so before it loaded what the stream saw last).
    uint64_t full[18], empty[9];
    uint64_t told[kSegments];
    uint64_t scores[2], taken[2], weights[2][2], half[2], done[2], queries, drained;   // by stream; weights by half of a tile
    int32_t pages_known[8];          // by tile: bits of its pages that are there (read before the eighth after it is loaded)
    uint32_t tmem;
    int32_t gave_up;                 // a wait ran out: everybody leaves
    uint64_t last[2];                // what was issued before leaving so
    union {
        Segment segment[kSegments];
        uint64_t stage[kAttnWarps][4];   // rings of record warps
    };
};

template <int D>
constexpr int kSharedBytes = Geo<D>::kData + (int)sizeof(Control);
static_assert(kSharedBytes<128> <= 232448 && kSharedBytes<64> <= 232448, "shared memory of a CTA");

__device__ __forceinline__ bool plan_fits(const PlanHeader& h, const AttnArgs& a, uint32_t magic = kPlanMagic)
{
    return h.magic == magic && h.batch == a.batch && h.hq == a.hq && h.hkv == a.hkv && h.dim == a.dim && h.grid == a.grid &&
           h.max_seqs == a.max_seqs && h.max_pages == a.max_pages;
}

// All lanes of a warp wait; false for all where it took too long or others gave up.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, Control& c, int32_t* err)
{
    const uint32_t addr = smem_addr(bar);
    if (__all_sync(0xffffffffu, mbar_try_wait(addr, parity))) return true;
    const long long t0 = clock64();
    while (true) {
        const bool ok = mbar_try_wait(addr, parity);
        const bool late = clock64() - t0 > kLimitCycles || *reinterpret_cast<volatile int32_t*>(&c.gave_up);
        if (__all_sync(0xffffffffu, ok)) return true;
        if (__any_sync(0xffffffffu, late)) {
            *reinterpret_cast<volatile int32_t*>(&c.gave_up) = 1;
            if ((threadIdx.x & 31) == 0) kv4_error(err, KVC_DEVERR_WAIT_TIMEOUT);
            return false;
        }
    }
}

__device__ __forceinline__ void arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

// ------------------------------------------------------------ large runs, tcgen05
// Both streams work on every tile (wide), or they take turns.  Tiles of K run ahead of those of V by two, so the ring's order within a segment is
// K 0 .. A - 1, then V n, K n + A, as far as there are any: where a tile lies in it.
struct Order {
    int ahead, tiles;
    __device__ __forceinline__ explicit Order(int n) : ahead(min(2, n)), tiles(n) {}
    __device__ __forceinline__ int k(int j) const { return j < ahead ? j : 2 * j - ahead + 1; }
    __device__ __forceinline__ int v(int n) const { return min(ahead + 2 * n, tiles + n); }
};
// A stream's tiles: how many, and its j-th.
__device__ __forceinline__ int stream_tiles(int tiles, bool wide, int stream) { return wide ? tiles : (tiles + 1 - stream) >> 1; }
__device__ __forceinline__ int stream_tile(bool wide, int stream, int j) { return wide ? j : 2 * j + stream; }

// Where a stream's scores lie in tensor memory, and its weights.  Wide: both streams' scores in the same 128 columns, so that those of the next
// tile can be made while this one's are worked (a softmax warp holds them in registers).  Else each has 128, and weights lie over scores.
__device__ __forceinline__ uint32_t scores_at(const Control& c, bool wide, int stream) { return c.tmem + (wide ? 0 : stream * 128); }
__device__ __forceinline__ uint32_t weights_at(const Control& c, bool wide, int stream) { return c.tmem + stream * (wide ? 64 : 128) + (wide ? 128 : 0); }

// The loading warp: goes through the worker's share segment by segment, tells the others of each and loads its tiles.
template <int D>
__device__ __forceinline__ void load_tiles(const AttnArgs& a, const CtaStart& start, Control& c, uint8_t* smem, const CUtensorMap* mk,
                                           const CUtensorMap* mv)
{
    using G = Geo<D>;
    const int lane = threadIdx.x & 31;
    const bool one = elect_one();
    const uint64_t policy = l2_policy_evict_first();
    uint32_t n = 0, tile_no = 0, told = 0;                // tiles of K and V so far; of both; segments
    auto tell = [&](const Segment& s) {
        if (lane == 0) {
            c.segment[told % kSegments] = s;
            arrive(&c.told[told % kSegments]);
        }
        ++told;
        __syncwarp();
    };
    Run r = start.r;
    Segment s = start.s;
    int run = start.run, job = start.job;
    bool fine = true;
    while (fine) {
        if (s.pages == 0) {                               // the next segment
            if (r.pages == 0 || job >= r.chunks * a.hkv) {
                run += r.pages == 0 ? 1 : r.rows;
                if (run >= a.batch) break;
                r = a.view.runs[run];
                job = 0;
                continue;
            }
            s = make_segment(r, run, job, 0, start.end, a.hkv, a.G, blockIdx.x);
            if (s.pages == 0) break;
            ++job;
        }
        tell(s);

        const int32_t* row = a.table + (int64_t)r.req * a.max_pages + s.first;
        const int tiles = s.tiles();
        const Order order(tiles);
        // Page ids: a lane has a page of a window of four tiles, and of the one before it (V comes up to two later).
        auto ids_of = [&](int window) {
            const int page = window * 32 + lane;
            return page < s.pages ? row[page] : -1;
        };
        int next = ids_of(0), now = -1, before = -1, kt = 0, vt = 0;
#pragma unroll 1
        for (int i = 0; i < 2 * tiles; ++i, ++n) {
            const bool of_k = kt < tiles && i == order.k(kt);
            if (of_k && kt % 4 == 0) {
                before = now;
                now = next;
                next = ids_of(kt / 4 + 1);
            }
            const int t = of_k ? kt++ : vt++;
            // (One lane issues the tile's copies, with operands in uniform registers: lanes with a copy each would be served one
            // after the other, some 130 cycles each, which bounded the whole kernel.)
            const int np = s.tile_pages(t), slot = n % G::kSlots, held = (kt - 1) / 4 == t / 4 ? now : before;
            const uint32_t bar = smem_addr(&c.full[n % (2 * G::kSlots)]), dst = smem_addr(smem + G::kRing + slot * G::kTileBytes);
            int rows[kTilePages];
            uint32_t mask = 0;
#pragma unroll
            for (int p = 0; p < kTilePages; ++p) {
                const int id = __shfl_sync(0xffffffffu, held, (t % 4) * kTilePages + p);
                mask |= (p < np && id >= 0 && id < a.num_pages ? 1u : 0u) << p;
                rows[p] = (id * a.hkv + s.head) * kPageSize;
            }
            if (!(fine = warp_wait(&c.empty[slot], (n / G::kSlots & 1) ^ 1, c, a.err))) break;
            if (one) {
                if (of_k) c.pages_known[(tile_no + t) % 8] = (int32_t)mask;
                if (mask != (1u << np) - 1u) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
                mbar_arrive_expect_tx(bar, __popc(mask) * (uint32_t)G::kPageBytes);
                const CUtensorMap* const map = of_k ? mk : mv;
#pragma unroll
                for (int p = 0; p < kTilePages; ++p)
                    if (mask >> p & 1u) {
#pragma unroll
                        for (int b = 0; b < G::kBlocks; ++b) tma_load_3d(dst + b * G::kBlockBytes + p * 2048, map, 0, rows[p], b, bar, policy);
                    }
            }
            __syncwarp();
        }
        tile_no += tiles;
        s.pages = 0;
    }
    if (fine) tell(s);
    // The CTA does not leave before its slots have been told to be free.
    for (uint32_t i = n > G::kSlots ? n - G::kSlots : 0; fine && i < n; ++i) fine = warp_wait(&c.empty[i % G::kSlots], i / G::kSlots & 1, c, a.err);
    // Where others gave up: what is under way arrives before the CTA leaves.
    if (*reinterpret_cast<volatile int32_t*>(&c.gave_up))
        for (uint32_t i = n > G::kSlots ? n - G::kSlots : 0; i < n; ++i)
            mbar_wait_bounded(smem_addr(&c.full[i % (2 * G::kSlots)]), i / (2 * G::kSlots) & 1, kLimitNs);
}

// A stream's issuing warp.  Wide: the scores of its next tile, as soon as the other stream has taken its own from the columns that they share, then
// the weights of the tile before against V, in halves as they come.  Else first a tile's weights against V, then the next one's scores.  (All of the warp goes along, so that addresses and descriptors stay in uniform
// registers; one lane issues.  Two warps, since what one does between its products takes as long as those.)
template <int D, class T, bool kWide>
__device__ __forceinline__ void issue_products(const AttnArgs& a, Control& c, uint8_t* smem, int stream)
{
    using G = Geo<D>;
    constexpr bool kBf16 = std::is_same_v<T, Bf16>;
    const uint32_t base = smem_addr(smem), ring = base + G::kRing, to = c.tmem + kOut + stream * 128;
    const bool one = elect_one();
    uint32_t n0 = 0, before = 0, others = 0, second_halves = 0;   // tiles of both; of this stream; of the other
#pragma unroll 1
    for (uint32_t segment = 0;; ++segment) {
        if (!warp_wait(&c.told[segment % kSegments], segment / kSegments & 1, c, a.err)) return;
        const Segment s = c.segment[segment % kSegments];
        if (s.pages == 0) return;
        const bool wide = kWide && s.wide;
        const int tiles = s.tiles(), mine = stream_tiles(tiles, wide, stream);
        const Order order(tiles);
        const uint64_t q = smem_desc(base + (wide ? stream * G::kQueryTile : 0), 16, 1024);
        const uint32_t vdesc = mma_desc(kBf16, true, kTileRows, D);
        auto arrived = [&](int at) { return warp_wait(&c.full[(n0 + at) % (2 * G::kSlots)], (n0 + at) / (2 * G::kSlots) & 1, c, a.err); };
        // A slot is free when the products that both streams, or the one that has the tile, issued with it are done.
        auto free_slot = [&](int at) {
            uint64_t* const slot = &c.empty[(n0 + at) % G::kSlots];
            mma_commit(smem_addr(slot));
            if (!wide) arrive(slot);
        };
        if (!warp_wait(&c.queries, segment & 1, c, a.err)) return;
        const uint32_t ts = scores_at(c, wide, stream), tp = weights_at(c, wide, stream);
        int j = 0, n = 0;                 // tiles whose scores, and whose products with V, have been issued
        while (n < mine) {
            if (j < mine && j <= n + wide) {
                const int t = stream_tile(wide, stream, j), at = order.k(t);
                const uint64_t k = smem_desc(ring + (n0 + at) % G::kSlots * G::kTileBytes, 16, 1024);
                const uint32_t kdesc = mma_desc(kBf16, false, kTileRows, s.tile_pages(t) * kPageSize);
                if (!arrived(at)) return;
                // (Where the streams share the columns their scores follow one another by turns; a segment's first find them free.)
                if (wide && (stream == 1 || j > 0) && !warp_wait(&c.taken[stream ^ 1], (others + j - (stream == 0)) & 1, c, a.err)) return;
                tmem_fence_after();
                if (one) {
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
                        mma_ss(ts, q + (((ks / 4) * G::kQueryBlock + (ks % 4) * 32) >> 4), k + (((ks / 4) * G::kBlockBytes + (ks % 4) * 32) >> 4),
                               kdesc, ks > 0);
                    mma_commit(smem_addr(&c.scores[stream]));
                    arrive(&c.scores[stream]);   // (what the loading warp has said of the tile comes along)
                    free_slot(at);
                }
                ++j;
            } else {
                const int t = stream_tile(wide, stream, n), at = order.v(t), pages = s.tile_pages(t);
                const uint64_t v = smem_desc(ring + (n0 + at) % G::kSlots * G::kTileBytes, G::kBlockBytes, 1024);
                if (!arrived(at)) return;
                if (!warp_wait(&c.weights[stream][0], (before + n) & 1, c, a.err)) return;
                tmem_fence_after();
                if (one) {
#pragma unroll
                    for (int kk = 0; kk < kTilePages / 2; ++kk)
                        if (kk < pages) mma_ts(to, tp + kk * 8, v + kk * (2048 >> 4), vdesc, n > 0 || kk > 0);
                    if (!kWide && pages > kTilePages / 2) mma_commit(smem_addr(&c.half[stream]));
                }
                __syncwarp();
                if (pages > kTilePages / 2) {
                    if (!warp_wait(&c.weights[stream][1], second_halves++ & 1, c, a.err)) return;
                    tmem_fence_after();
                }
                if (one) {
#pragma unroll
                    for (int kk = kTilePages / 2; kk < kTilePages; ++kk)
                        if (kk < pages) mma_ts(to, tp + kk * 8, v + kk * (2048 >> 4), vdesc, true);
                    mma_commit(smem_addr(&c.done[stream]));
                    free_slot(at);
                }
                ++n;
            }
            __syncwarp();
        }
        if (mine == 0 && one) arrive(&c.done[stream]);   // (the stream's softmax goes on with its issuing warp)
        __syncwarp();
        before += mine;
        others += stream_tiles(tiles, wide, stream ^ 1);
        n0 += 2 * tiles;
    }
}

// The segment's queries, by the softmax warps: 16-byte chunks of up to 256 rows into the tiles' swizzle, all under way at once.
template <int D>
__device__ __forceinline__ void load_queries(const AttnArgs& a, const Segment& s, uint8_t* smem)
{
    using G = Geo<D>;
    constexpr int kChunks = D / 8, kStep = 32 * kSoftmaxWarps / kChunks;   // chunks of a row; rows at a time
    const int total = s.rows * a.G, ch = threadIdx.x % kChunks, rows0 = s.rows0 * a.G;
    const uint32_t by = (65536u + a.G - 1) / a.G;           // qr / G = qr * by >> 16 for qr < 256, G <= 8
    const uint16_t* q = a.q + (int64_t)s.row0 * a.q_stride + (int64_t)s.head * a.G * D + ch * 8;
    const uint32_t to = smem_addr(smem) + (ch >> 3) * G::kQueryBlock;
#pragma unroll 2
    for (int qr = threadIdx.x / kChunks; qr < total; qr += kStep) {
        const int br = (int)(qr * by >> 16), tile = qr >= rows0, r = qr - (tile ? rows0 : 0);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + tile * G::kQueryTile + r * 128 + (((ch & 7) ^ (r & 7)) << 4)),
                     "l"(q + br * a.q_stride + (int64_t)(qr - br * a.G) * D)
                     : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// Bits of a page's 16 tokens that take part: none of a page that is not there, of the last page those before the prefix's end
// (valid: the tile's tokens before it).
__device__ __forceinline__ uint32_t token_bits(int page, uint32_t known, int valid)
{
    const int n = min(max(valid - page * kPageSize, 0), kPageSize);
    return known >> page & 1u ? (1u << n) - 1u : 0u;
}

__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return d;
}

// The softmax of a thread's row over N x 32 tokens whose scores are x.
template <int D, class T>
struct RowSoftmax {
    float top = -INFINITY, l = 0.f;   // reference, as a score; the sum of weights
    float sub = -Weights<T>::kShift;  // what weigh() takes off scores in log2 units
    bool far = false;                 // a row of this warp's is far out

    // The reference in log2 units, and whether it is far out.
    __device__ __forceinline__ float reference(float sl) const { return __fmul_rn(top, sl); }
    __device__ __forceinline__ bool is_far(float sl) const { return fabsf(reference(sl)) >= kFar && top != -INFINITY; }

    // Tokens that do not take part: bits of 16 for each page.
    template <int N>
    static __device__ __forceinline__ void mask(uint32_t (&x)[N][32], int page, uint32_t known, int valid)
    {
#pragma unroll
        for (int w = 0; w < N; ++w) {
            const uint32_t bits = token_bits(page + 2 * w, known, valid) | token_bits(page + 2 * w + 1, known, valid) << 16;
#pragma unroll
            for (int i = 0; i < 32; ++i) x[w][i] = bits >> i & 1u ? x[w][i] : 0xff800000u;
        }
    }
    // Whether the reference has to move, and where to: a score exceeds it by more than 8 in log2 units (see the top).
    template <int N>
    __device__ __forceinline__ bool exceeds(const uint32_t (&x)[N][32], float sl, float* to) const
    {
        float y[8];                                       // (eight chains)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fmaxf(__uint_as_float(x[0][i]), __uint_as_float(x[1][i]));
#pragma unroll
        for (int i = 8; i < 32; ++i) y[i & 7] = max3(__float_as_uint(y[i & 7]), x[0][i], x[1][i]);
#pragma unroll
        for (int w = 2; w < N; w += 2)
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i & 7] = max3(__float_as_uint(y[i & 7]), x[w][i], x[w + 1][i]);
#pragma unroll
        for (int d = 4; d > 0; d >>= 1)
#pragma unroll
            for (int i = 0; i < d; ++i) y[i] = fmaxf(y[i], y[i + d]);
        *to = y[0];
        return (y[0] - top) * sl > 8.f;
    }
    // It moves, and with it the sums so far, in whose columns nothing is under way (none: there are no sums yet).
    __device__ __forceinline__ void move(bool moves, float to, float sl, bool none, uint32_t out)
    {
        if (!none) {
            const float is = __fmul_rn(to, sl);
            const float alpha = moves ? ex2(fabsf(is) >= kFar ? (top - to) * sl : reference(sl) - is) : 1.f;
            l *= alpha;
#pragma unroll 1
            for (int w = 0; w < D / 16; ++w) {
                uint32_t o[16];
                tmem_ld16(out + 16 * w, o);
                tmem_wait_ld();
                tmem_loaded(o);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                tmem_st16(out + 16 * w, o);
            }
        }
        top = moves ? to : top;
        sub = (is_far(sl) || top == -INFINITY ? 0.f : reference(sl)) - Weights<T>::kShift;
        far = __any_sync(0xffffffffu, is_far(sl));
    }
    // Weights come from one fused multiply-add of score, scale and the reference in log2 units, whose rounding is the same for all weights
    // and for m.  Far out, where it counts, the reference is taken off the scores first.
    template <int N>
    __device__ __forceinline__ void approach(uint32_t (&x)[N][32], float sl) const
    {
        const float by = is_far(sl) ? top : 0.f;
#pragma unroll
        for (int w = 0; w < N; ++w)
#pragma unroll
            for (int i = 0; i < 32; ++i) x[w][i] = __float_as_uint(__uint_as_float(x[w][i]) - by);
    }
    // Weights of 32 tokens, in the pool's type, and their sum.
    __device__ __forceinline__ void weigh(const uint32_t (&x)[32], float sl, uint32_t (&p)[16])
    {
        const uint64_t sl2 = f2_pack(sl, sl), sub2 = f2_pack(-sub, -sub);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float u, v;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), sl2, sub2), u, v);
            u = ex2(u);
            v = ex2(v);
            sum[i & 1] = f2_add(sum[i & 1], f2_pack(u, v));
            p[i] = T::pack(u, v);
        }
        float u, v;
        f2_unpack(f2_add(sum[0], sum[1]), u, v);
        l += u + v;
    }
};

// A stream's softmax: a thread owns a row of the tile.
template <int D, class T, bool kWide>
__device__ __forceinline__ void softmax_stream(const AttnArgs& a, Control& c, uint8_t* smem)
{
    using G = Geo<D>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, stream = warp >> 2, wq = warp & 3;
    const int my = wq * 32 + lane;                        // row of the stream's tile
    const uint32_t quarter = (uint32_t)wq << 21, to = c.tmem + quarter + kOut + stream * 128;
    uint32_t n0 = 0, tile_no = 0, scored = 0, halves = 0, used = 0;   // phases of the stream's scores, half and done
    const float sl = a.scale_log2;
#pragma unroll 1
    for (uint32_t segment = 0;; ++segment) {
        if (!warp_wait(&c.told[segment % kSegments], segment / kSegments & 1, c, a.err)) return;
        const Segment& s = c.segment[segment % kSegments];
        if (s.pages == 0) return;
        if (segment > 0 && !warp_wait(&c.drained, (segment - 1) & 1, c, a.err)) return;
        load_queries<D>(a, s, smem);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) arrive(&c.queries);
        const bool wide = kWide && s.wide;
        const int tiles = s.tiles(), mine = stream_tiles(tiles, wide, stream);
        const int qrows = (wide && stream == 1 ? s.rows - s.rows0 : s.rows0) * a.G;
        const bool works = wq * 32 < qrows;               // (the others have no row of the tile)
        const Order order(tiles);
        const uint32_t ts = scores_at(c, wide, stream) + quarter, tp = weights_at(c, wide, stream) + quarter;
        RowSoftmax<D, T> row;
#pragma unroll 1
        for (int j = 0; j < mine; ++j) {
            const int t = stream_tile(wide, stream, j), pages = s.tile_pages(t), valid = s.valid - t * kTilePages * kPageSize;
            if (!warp_wait(&c.scores[stream], scored++ & 1, c, a.err)) return;
            tmem_fence_after();
            uint32_t x[kWide ? 4 : 1][32];
            if constexpr (kWide) {
                // All of the tile's scores into registers, and the columns are the other stream's.
                if (works) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) tmem_ld32(ts + 32 * w, x[w]);
                    tmem_wait_ld();
#pragma unroll
                    for (int w = 0; w < 4; ++w) tmem_loaded(x[w]);
                }
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) arrive(&c.taken[stream]);
            }
            const uint32_t known = (uint32_t)c.pages_known[(tile_no + t) % 8];
            const bool whole = valid >= kTilePages * kPageSize && known == (1u << kTilePages) - 1u;
            // Weights of a half are handed on at once: the first half's product with V runs while the second is worked.
            const int parts = pages > kTilePages / 2 ? 2 : 1;
            auto hand_on = [&](int h) {
                if (!whole) {   // rows of V that hold anything: zero, or 0 * NaN would reach the sums
                    const uint32_t n = n0 + order.v(t), vslot = n % G::kSlots;
                    if (!warp_wait(&c.full[n % (2 * G::kSlots)], n / (2 * G::kSlots) & 1, c, a.err)) return false;
#pragma unroll 1
                    for (int page = h * (kTilePages / 2); page < min(pages, (h + 1) * (kTilePages / 2)); ++page) {
                        const int from = known >> page & 1u ? valid - page * kPageSize : 0;   // (a thread has 16 bytes of each block)
                        if (my >> 3 >= from)
                            for (int b = 0; b < G::kBlocks; ++b)
                                *reinterpret_cast<uint4*>(smem + G::kRing + vslot * G::kTileBytes + b * G::kBlockBytes + page * 2048 + my * 16) =
                                    make_uint4(0u, 0u, 0u, 0u);
                    }
                    fence_proxy_async_smem();
                }
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) arrive(&c.weights[stream][h]);
                return true;
            };
            if constexpr (kWide) {
                uint32_t p[16];
                float mx;
                if (works) {
                    if (!whole) row.mask(x, 0, known, valid);
                    const bool moves = my < qrows && row.exceeds(x, sl, &mx);   // (no row looks at another's)
                    if (__any_sync(0xffffffffu, moves)) {
                        if (j > 0) {
                            if (!warp_wait(&c.done[stream], used & 1, c, a.err)) return;
                            tmem_fence_after();
                        }
                        row.move(moves, mx, sl, j == 0, to);
                    }
                    if (__builtin_expect(row.far, false)) row.approach(x, sl);
                    row.weigh(x[0], sl, p);
                }
                // Weights lie where those of the tile before did, when these have met V (where the streams take turns, before these
                // scores were made).
                if (wide && j > 0) {
                    if (!warp_wait(&c.done[stream], used & 1, c, a.err)) return;
                    tmem_fence_after();
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (h == parts) break;
                    if (works) {
                        if (h > 0) row.weigh(x[2], sl, p);
                        tmem_st16(tp + 32 * h, p);
                        row.weigh(x[2 * h + 1], sl, p);
                        tmem_st16(tp + 32 * h + 16, p);
                        tmem_wait_st();
                    }
                    if (!hand_on(h)) return;
                }
            } else {
                // A half at a time all along: fewer instructions to fetch, and weights sooner, where there are few tiles.  (Scores that
                // have come were made after the products of the tile before.)
#pragma unroll 1
                for (int h = 0; h < parts; ++h) {
                    if (works) {
                        uint32_t x[2][32], p[16];
                        float mx;
                        tmem_ld32(ts + 64 * h, x[0]);
                        tmem_ld32(ts + 64 * h + 32, x[1]);
                        tmem_wait_ld();
                        tmem_loaded(x[0]);
                        tmem_loaded(x[1]);
                        if (!whole) row.mask(x, 4 * h, known, valid);
                        const bool moves = my < qrows && row.exceeds(x, sl, &mx);
                        if (__any_sync(0xffffffffu, moves)) {
                            if (h > 0) {
                                if (!warp_wait(&c.half[stream], halves & 1, c, a.err)) return;
                                tmem_fence_after();
                            }
                            row.move(moves, mx, sl, j == 0 && h == 0, to);
                        }
                        if (__builtin_expect(row.far, false)) row.approach(x, sl);
                        row.weigh(x[0], sl, p);
                        tmem_st16(tp + 32 * h, p);
                        row.weigh(x[1], sl, p);
                        tmem_st16(tp + 32 * h + 16, p);
                        tmem_wait_st();
                    }
                    if (!hand_on(h)) return;
                }
                halves += parts - 1;
            }
            used += j > 0;
        }
        const bool some = mine > 0;
        if (!warp_wait(&c.done[stream], used++ & 1, c, a.err)) return;   // (the last products are in)
        if (lane == 0) arrive(&c.drained);                              // (this stream's products need the queries no more)
        n0 += 2 * tiles;
        tile_no += tiles;
        tmem_fence_after();
        if (works) {
            // A row's results, 32 bytes (a sector) of each at a time.  (By way of shared memory, so that a row's columns leave together: d = 64 4 %
            // longer, four rows on an image 9.2 us a layer instead of 8.8, one prefix of 32768 tokens 27.1 instead of 27.5.)
            const int64_t entry = s.entry + (stream == 0 ? 0 : s.rows0 * a.G);
            if (my < qrows) a.view.run_ml[entry + my] = make_float2(some ? row.reference(sl) : -INFINITY, some ? row.l : 0.f);
            float* const row_o = a.view.run_o + (entry + my) * D;
#pragma unroll 1
            for (int w = 0; some && w < D / 32; ++w) {
                uint32_t o[32];
                tmem_ld32(to + 32 * w, o);
                tmem_wait_ld();
                tmem_loaded(o);
                if (my < qrows) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row_o + 32 * w + 8 * i), "r"(o[8 * i]), "r"(o[8 * i + 1]),
                                     "r"(o[8 * i + 2]), "r"(o[8 * i + 3]), "r"(o[8 * i + 4]), "r"(o[8 * i + 5]), "r"(o[8 * i + 6]), "r"(o[8 * i + 7])
                                     : "memory");
                }
            }
        }
        tmem_fence_before();
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
        r = s.r;
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
__device__ __forceinline__ void work_records(const AttnArgs& a, const WarpStart& start, Control& c, uint8_t* smem, const CUtensorMap* mk,
                                             const CUtensorMap* mv)
{
    using G = Geo<D>;
    constexpr int KS = D / 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (start.count == 0) return;
    const int worker = start.worker;
    int left = start.count;
    uint8_t* const ring = smem + warp * G::kWarpRing;
    if (lane < G::kStages) mbar_init(smem_addr(&c.stage[warp][lane]), 1);
    fence_mbar_init();
    __syncwarp();
    const uint64_t policy = l2_policy_evict_first();

    // The ring's side: a page's K and V by lanes of 64 columns each.
    Windows win(a, start, left);
    uint32_t skipped = 0, phase = 0;                 // bits by stage: a page that is not there; the barrier's parity
    int put = 0, staged = 0;
    const bool one = elect_one();
    auto load = [&] {
        if (win.done()) return;
        const int id = win.id();
        const bool known = id >= 0 && id < a.num_pages;
        const uint32_t bar = smem_addr(&c.stage[warp][put]);
        if (known) {
            skipped &= ~(1u << put);
            if (one) {
                const uint32_t dst = smem_addr(ring + put * 2 * G::kPageBytes);
                const int row = (id * a.hkv + win.cur_head) * kPageSize;
                mbar_arrive_expect_tx(bar, 2 * G::kPageBytes);
#pragma unroll
                for (int b = 0; b < G::kBlocks; ++b) {
                    tma_load_3d(dst + b * 2048, mk, 0, row, b, bar, policy);
                    tma_load_3d(dst + G::kPageBytes + b * 2048, mv, 0, row, b, bar, policy);
                }
            }
            __syncwarp();
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
    Record r = start.r;
    while (left > 0 && fine) {
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
                for (int k = 0; k < 4; ++k) sc[k] = __fmul_rn(acc[0][k] + acc[1][k], a.scale_log2);   // (not fused with the difference below)
                // Lane: tokens lane / 4 and + 8, columns 2 (lane % 4) and + 1.
                const int t0 = lane >> 2;
                if (valid < kPageSize) {
                    if (t0 >= valid) sc[0] = sc[1] = -INFINITY;
                    if (t0 + 8 >= valid) sc[2] = sc[3] = -INFINITY;
                }
                const float x0 = fmaxf(sc[0], sc[2]), x1 = fmaxf(sc[1], sc[3]);
                if (__any_sync(0xffffffffu, x0 - m0 > 8.f || x1 - m1 > 8.f)) {
                    float y0 = x0, y1 = x1;
#pragma unroll
                    for (int k = 4; k < 32; k <<= 1) {
                        y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, k));
                        y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, k));
                    }
                    const bool moves0 = y0 - m0 > 8.f, moves1 = y1 - m1 > 8.f;   // (no column looks at another's)
                    const float f0 = moves0 ? ex2(m0 - y0) : 1.f, f1 = moves1 ? ex2(m1 - y1) : 1.f;
                    m0 = moves0 ? y0 : m0;
                    m1 = moves1 ? y1 : m1;
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
                constexpr float kShift = Weights<T>::kShift;
                const float s0 = m0 == -INFINITY ? 0.f : m0, s1 = m1 == -INFINITY ? 0.f : m1;
                const float p0 = ex2(sc[0] - s0 + kShift), p1 = ex2(sc[1] - s1 + kShift), p2 = ex2(sc[2] - s0 + kShift), p3 = ex2(sc[3] - s1 + kShift);
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
        const int64_t entry = record_entry(r.col, r.rows, a.hkv, a.G, head, worker);
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
            if (lane < 4) a.view.rec_ml[entry + cc] = make_float2(k ? m1 : m0, k ? l1 : l0);
        }
        // The next job.
        if (left > 0) {
            page = 0;
            if (++head == a.hkv) {
                head = 0;
                do r = a.view.recs[++rec];
                while (r.pages == 0);
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

// kWide: for batches of more than 128 query rows of a KV head, whose runs may have more than a stream holds.  The other kernel has half the softmax's
// instructions to fetch, which shows where a CTA has a tile or two: four rows of 28/4 heads on 1369 tokens take 9.0 us a layer with it, 9.2 with this one.
// (This one against that, when that still took such batches: 131009 tokens and 96 rows 151 against 173, 32768 and 32 rows 27.1 against 29.6, eleven
// small groups at d = 64 23.7 against 22.8.)
template <int D, class T, bool kWide>
__global__ void __launch_bounds__(kThreads, 1) attention_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                                                                const __grid_constant__ AttnArgs a)
{
    // (The kernel has no other shared memory: what it is given starts on 1024 bytes, as the swizzle wants it.)
    extern __shared__ __align__(1024) uint8_t smem[];
    Control& c = *reinterpret_cast<Control*>(smem + Geo<D>::kData);
    const int tid = threadIdx.x, warp = tid >> 5;
    if (tid < 18) mbar_init(smem_addr(&c.full[tid]), 1);
    if (tid < 9) mbar_init(smem_addr(&c.empty[tid]), 2);
    if (tid >= 64 && tid < 64 + kSegments) mbar_init(smem_addr(&c.told[tid - 64]), 1);
    if (tid < 2) {
        mbar_init(smem_addr(&c.scores[tid]), 2);
        mbar_init(smem_addr(&c.half[tid]), 1);
        mbar_init(smem_addr(&c.taken[tid]), 4);
        mbar_init(smem_addr(&c.done[tid]), 1);
    }
    if (tid < 4) mbar_init(smem_addr(&c.weights[0][0] + tid), 4);
    if (tid == 2) mbar_init(smem_addr(&c.queries), kSoftmaxWarps);
    if (tid == 3) mbar_init(smem_addr(&c.drained), kSoftmaxWarps);
    if (tid == 4) c.gave_up = 0;
    if (tid == 5 || tid == 6) mbar_init(smem_addr(&c.last[tid - 5]), 1);
    if (tid == 0) {
        prefetch_tensormap(&mk);
        prefetch_tensormap(&mv);
    }
    // Tensor memory for all (it is given back at once where the CTA turns out to work on records): while the launch before
    // finishes this costs nothing.
    if (warp == kMmaWarp) tmem_alloc(smem_addr(&c.tmem), 512);
    fence_mbar_init();
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    griddep_wait();
    griddep_launch_dependents();
    const PlanHeader h = *a.view.header;
    // (What either kind of CTA starts with comes along with the header; the other's is not looked at.)
    const WarpStart mine = a.view.warp_starts[blockIdx.x * kAttnWarps + warp];
    CtaStart start;
    if (warp == kLoadWarp) start = a.view.cta_starts[blockIdx.x];
    const bool fits = plan_fits(h, a) && (smem_addr(smem) & 1023) == 0, records = (int)blockIdx.x >= h.prefix_ctas;
    if (!fits || records) {
        if (warp == kMmaWarp) tmem_dealloc(c.tmem, 512);
        if (!fits) {
            if (tid == 0 && blockIdx.x == 0) kv4_error(a.err, plan_fits(h, a, kPlanGaveUp) ? KVC_DEVERR_WAIT_TIMEOUT : KVC_DEVERR_PLAN);
            return;
        }
        work_records<D, T>(a, mine, c, smem, &mk, &mv);
        if (*reinterpret_cast<volatile int32_t*>(&c.gave_up)) a.view.header->magic = kPlanGaveUp;
        return;
    }
    if (warp < kSoftmaxWarps) {
        if constexpr (kWide) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegisters));
        softmax_stream<D, T, kWide>(a, c, smem);
    } else {
        if constexpr (kWide) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
        if (warp == kLoadWarp) {
            load_tiles<D>(a, start, c, smem, &mk, &mv);
        } else if (warp < kMmaWarp + 2) {
            issue_products<D, T, kWide>(a, c, smem, warp - kMmaWarp);
            if (*reinterpret_cast<volatile int32_t*>(&c.gave_up) && elect_one()) {   // what is under way ends before the memory is freed
                uint64_t* const last = &c.last[warp - kMmaWarp];
                mma_commit(smem_addr(last));
                mbar_wait_bounded(smem_addr(last), 0, kLimitNs);
            }
            __syncwarp();
        }
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    if (warp == kMmaWarp) tmem_dealloc(c.tmem, 512);
    if (tid == 0 && c.gave_up) a.view.header->magic = kPlanGaveUp;
}

// ---------------------------------------------------------------------- merge
// A CTA of four warps per (row, query head): the partial results of the row's own segments, then its prefix's, in their order.
// Each warp takes every fourth; with loads of eight under way, a unit of up to 32 segments is one trip to L2 after its sources.  Bound by
// those trips and the launch: 1.3 us behind the attention of one row, 3.5 us for 896 units of 33 segments each (15 MB).
template <int D, class T>
__global__ void __launch_bounds__(128) merge_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr int N = D / 32;
    using Vec = std::conditional_t<N == 4, float4, float2>;
    __shared__ float s_o[4][D];
    __shared__ float2 s_ml[4];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int head = blockIdx.x, row = blockIdx.y;
    const int kv = (int)((uint32_t)head * ((65536u + a.G - 1) / a.G) >> 16), g = head - kv * a.G;   // (head < 8192, G <= 8)
    const RowSources x = a.view.rows[(int64_t)row * a.hkv + kv];
    const PlanHeader h = *a.view.header;
    if (!plan_fits(h, a)) {
        if (plan_fits(h, a, kPlanGaveUp)) {           // partial results are not all there, or those of another call
            for (int i = threadIdx.x; i < D; i += 128) a.out[(int64_t)row * a.out_stride + (int64_t)head * D + i] = (uint16_t)T::pack(NAN, NAN);
            if (a.lse && threadIdx.x == 0) a.lse[(int64_t)row * a.hq + head] = NAN;
        }
        return;
    }
    const int own = x.own_count, total = own + x.prefix_count;
    const bool run = x.stream_step >= 0;

    float m = -INFINITY, l = 0.f, o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.f;
#pragma unroll 1
    for (int s0 = warp; s0 < total; s0 += 128) {
        // This lane's segment: its (m, l) and where its sums lie.
        const int s = s0 + 4 * lane, n = min(32, (total - s0 + 3) / 4), p = s - own;
        const bool in_run = run && p >= 0;
        const int64_t e = g + (p < 0                 ? x.own + (int64_t)s * kRecordCols
                               : x.stream_step > 0 ? x.prefix + (int64_t)(p >> 1) * x.step + (p & 1 ? x.stream_step : 0)
                                                   : x.prefix + (int64_t)p * x.step);
        const float2 ml = lane < n ? (in_run ? a.view.run_ml : a.view.rec_ml)[e] : make_float2(-INFINITY, 0.f);
        const uint64_t from = reinterpret_cast<uint64_t>((in_run ? a.view.run_o : a.view.rec_o) + e * D);
        // The first eight's sums come along with them.
        Vec v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) v[j] = reinterpret_cast<const Vec*>(__shfl_sync(0xffffffffu, from, j))[lane];
        float top = ml.y == 0.f ? -INFINITY : ml.x;   // (a segment without tokens has no part)
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        top = fmaxf(top, m);
        const float old = m == top ? 1.f : ex2(m - top), mine = ml.y == 0.f ? 0.f : ml.x == top ? 1.f : ex2(ml.x - top);
        float sum = ml.y * mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        m = top;
        l = l * old + sum;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] *= old;
        float f[8];
        auto add = [&] {                              // (what has no weight may hold anything)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (f[j] != 0.f) {
                    o[0] += f[j] * v[j].x;
                    o[1] += f[j] * v[j].y;
                    if constexpr (N == 4) {
                        o[2] += f[j] * v[j].z;
                        o[3] += f[j] * v[j].w;
                    }
                }
            }
        };
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __shfl_sync(0xffffffffu, mine, j);
        add();
        uint32_t parts = __ballot_sync(0xffffffffu, mine != 0.f) & ~0xffu;
        while (parts) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int k = parts ? __ffs(parts) - 1 : 0;
                f[j] = __shfl_sync(0xffffffffu, mine, k);
                if (!parts) f[j] = 0.f;
                else v[j] = reinterpret_cast<const Vec*>(__shfl_sync(0xffffffffu, from, k))[lane];
                parts &= parts - 1;
            }
            add();
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) s_o[warp][lane * N + i] = o[i];
    if (lane == 0) s_ml[warp] = make_float2(m, l);
    __syncthreads();
    if (warp != 0) return;
    float f[4], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, s_ml[k].y == 0.f ? -INFINITY : s_ml[k].x);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 ml = s_ml[k];
        f[k] = ml.y == 0.f ? 0.f : ml.x == top ? 1.f : ex2(ml.x - top);
        sum += f[k] * ml.y;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float y = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) y += f[k] * s_o[k][lane * N + i];
        // (An average of numbers at the end of the range, taken with rounded weights, may pass it.)
        y *= inv;
        o[i] = fabsf(y) < INFINITY ? fminf(fmaxf(y, -Weights<T>::kMost), Weights<T>::kMost) : y;
    }
    uint16_t* const dst = a.out + (int64_t)row * a.out_stride + (int64_t)head * D + lane * N;
    if constexpr (N == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(T::pack(o[0], o[1]), T::pack(o[2], o[3]));
    else *reinterpret_cast<uint32_t*>(dst) = T::pack(o[0], o[1]);
    if (a.lse && lane == 0) a.lse[(int64_t)row * a.hq + head] = sum == 0.f ? -INFINITY : top * 0.693147180559945309f + logf(sum * exp2f(-Weights<T>::kShift));
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

template <int D, class T, bool kWide>
int launch_attention(const CUtensorMap& mk, const CUtensorMap& mv, const AttnArgs& a, cudaStream_t st)
{
    const auto kernel = attention_kernel<D, T, kWide>;
    static OncePerDevice once;                        // (what fails is tried again by the next call)
    int device = 0;
    if (cudaError_t e = cudaGetDevice(&device); e != cudaSuccess) return kv4_launch_result(e);
    const cudaError_t ready = once(device, [&] {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes<D>);
        if (e != cudaSuccess || !kWide) return e;
        return enough_registers(kSoftmaxWarps + 4, kMovedRegisters, [&](int* n) {
            cudaFuncAttributes f{};
            const cudaError_t asked = cudaFuncGetAttributes(&f, kernel);
            *n = f.numRegs;
            return asked;
        });
    });
    if (ready != cudaSuccess) return kv4_launch_result(ready);
    if (cudaError_t e = kv4_launch(kernel, dim3((unsigned)a.grid), kThreads, kSharedBytes<D>, st, mk, mv, a); e != cudaSuccess)
        return kv4_launch_result(e);
    return kv4_launch_result(kv4_launch(merge_kernel<D, T>, dim3((unsigned)a.hq, (unsigned)a.batch), 128, 0, st, a));
}

template <int D, class T>
int launch_attention(const CUtensorMap& mk, const CUtensorMap& mv, const AttnArgs& a, cudaStream_t st)
{
    return a.batch * a.G > kTileRows ? launch_attention<D, T, true>(mk, mv, a, st) : launch_attention<D, T, false>(mk, mv, a, st);
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
