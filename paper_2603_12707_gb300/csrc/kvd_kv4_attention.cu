// kv4_decode_attention: single-token decode attention over the 4-bit paged
// cache (layout: kvdecode4.h).
//
// With K_td = s_t (c_td - 8) + z_t and V_td = s'_t (c'_td - 8) + z'_t over the
// elements d of a scale group, a query row n (scaled to log2 units) has
//
//     S_tn = sum_groups s_t * sum_d q_nd (c_td - 8) + z_t * sum_d q_nd
//     o_nd = sum_t (p_tn s'_t) (c'_td - 8) + sum_t p_tn z'_t,   p_tn = 2^(S_tn - m_n)
//
// so scales and middles multiply scores and weights, 16 per page, and the codes
// go into the tensor cores as they are: a 4-bit code under a mask is an fp16
// subnormal, or nearly one, c * 2^-24 in bits 0-3 and c * 2^-20 in bits 4-7 (up to
// bit 10 a word's value is its bits), whose product with another fp16 is exact.  Eight of
// V's codes take five instructions to become four operands, of K's six.  The other
// operand is q, scaled by a power of two into fp16's range (and by what its codes' place
// asks), or p * s', relative to a power of two 2^E that follows the largest of them: one for each
// query head and scale group, so that neither another group's scales, nor another head's tokens, nor wide
// tokens of no weight take bits away (one E of the largest s' alone: a token of 2^40 times the others'
// scale and e^-90 of their weight moved outputs by 0.35).
//
// The tensor cores cut what they add off toward zero, and the products of a
// subnormal the earlier the smaller it is.  So K's codes are moved up by three bits
// (relative error of one token's score, rms: 2.4e-7 with an fp16 q, 2.1e-6 where they lie; 64
// MHA rows 56.0 -> 57.0 us).  For V it is a share of the sum that shows where a long row's outputs are
// small, and the codes' 8 is subtracted by one more product of the same rounded
// p * s' with constant rows that lose as much: the middle of the codes as the codes lie
// (120 for bits 4-7; 15 for bits 0-3, whose 7.5 is no fp16).
// Rows of -8 left 2.7e-4 of the mean output missing at 32K tokens; these 8e-5.
// What is lost all the same is of one sign and grows with the running sum, so after every 32 tiles
// of a row its sums go from the tensor cores' accumulators to fp32 ones, which are rounded to nearest, and
// begin anew: fp16 outputs of flat weights are 3.1e-4 off where a warp works 57, 256, 1024 or 2048
// pages of a row (2.1e-4 of it is their own rounding); in one sum 3.1e-4, 9.9e-4, 1.2e-2 and 2.8e-2.
// For K the 8 is in sum_groups (z - 8 s) sum q, a product of the scale words as they lie.
//
// Schedule.  The work is the list of all (row, KV head, page) tiles, a row's
// heads in turn and a head's pages in order.  Every warp of a persistent grid
// takes a consecutive share of equal cost, found from a scan over the rows'
// lengths in shared memory: no plan, no host lengths, and rows of any
// raggedness give equal shares.  A tile is one consecutive block of the pool,
// streamed by one bulk copy into the warp's ring of shared memory; K is the
// MMA's 16-row operand (its rows are the 16 tokens of the page), V^T's rows are
// elements, the G <= 8 query heads are the 8 columns of both.
//
// A (row, KV head) that lies in one warp's share is written by that warp.
// Others leave (o, m, l) per warp in shared memory, where the CTA merges what
// it holds; what crosses CTAs goes through the workspace to a second launch, in
// place when the first ends (a counter whose last CTA merges takes longer: one row
// of 32K tokens 22.8 us against 17, 64 rows of 32 KV heads 57.0 against 55.3).
//
// Roundings to fewer than 32 bits.  q and p * s' are fp16 operands, 11 bits: as many
// as fp16's own values, more than bf16's (a bf16 q
// loses only what is below 2^-35 of its row's largest, p * s' below 2^-31 of the largest in its sum).  sum q is 2 (fp16) or 3 (bf16) terms.  All
// sums, m, l and parts are fp32.  Against 64 bits, outputs over 32K tokens are
// 2.9e-4 off in fp16, of which 2.1e-4 are the output's own rounding, and 1.7e-3 in bf16, all of it that.
//
// Measured (device, calls in a graph; 6.8 TB/s is a copy's rate).  64 rows of 640 - 1344
// tokens, 32 KV heads, d 128: 60.3 us, 288 MB, 4.8 TB/s; 8 rows of 32K tokens,
// 28 query on 4 KV heads, groups of 32: 42.7 us, 168 MB, 3.9 TB/s; one row of 2337: 9.8 us.
// A further byte costs 1 / 6.1 TB/s (groups of 128), 5.5 (64), 5.5 (32), 5.3 (d 64): close
// to memory, beside which a tile's 290 to 406 instructions keep the ALU 56 % and
// the tensor cores 31 % busy.  What is left is fixed, some 13 us a call: the
// scan and the search 2.5, first tiles 1, the end of the shares and the CTA's merge 3, the
// second launch 2 to 3, and that a launch fetches its instructions anew (loops stay
// rolled and every large part has one call site: 74 KB -> 53 KB of code took one short row from 15.8 to 10.6 us).
#include <cmath>
#include <type_traits>

#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr uint64_t kWaitLimitNs = 1000000000ull;
constexpr float kLn2 = 0.6931471805599453f;
// What starting and ending a (row, KV head) costs a warp, in tiles: shares count it
// (64 rows of 0 - 8192 tokens, log-uniform: 55 us, 115 where shares are tiles alone).
constexpr uint32_t kRowCost = 3;
// What a warp takes at least, in tiles: a small call uses fewer warps rather than merge more parts.
constexpr uint32_t kMinShare = 2;
// Warps of a CTA that work at least, where there is enough for them: one per scheduler.
constexpr uint32_t kMinWarps = 4;

// A (row, KV head) that begins in a CTA and goes on in others (b < 0: there is none).
struct PartSpan {
    int32_t b, h, last;   // the last CTA that holds a part of it
    int32_t unused;
};

struct AttnArgs {
    const uint8_t* pool;
    int64_t num_pages;
    int32_t H, Hq, G;
    uint32_t H_inv;      // 2^32 / H, rounded down (2^32 - 1 for 1)
    uint32_t G_inv;      // 2^16 / G, rounded up
    const int32_t* block_table;
    const int32_t* lens;
    int32_t max_seqs, max_pages, batch;
    const int32_t* seq_ids;
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    float* lse;
    float scale;         // softmax scale * log2(e) * 2^21 (the accumulators' unit)
    PartSpan* spans;     // [grid]: what goes on after a CTA
    uint32_t* sums;      // [2][batch + 1] where shared memory does not hold them: the same from every CTA
    float* parts;        // [grid][2][G][D + 2]: a CTA's part of the row that began before it, and of the one that goes on
    int32_t* err;
};

// The shape of a variant: warps of the one CTA per SM (with two CTAs the older
// one's warps are served first, and half the SM idles while the other ends: 64
// MHA rows 5 us more; 12 warps where four groups' accumulators take more than 128
// registers, which cost the others 3 to 12 %), stages of a warp's ring (a third one is
// worth +0.5 % to -2 %), tiles of a stage, which a warp works together (four at d = 64:
// 5.6 against 4.9 TB/s; two at d = 128, where four do not fit).
template <int D, int NG>
struct AttnShape {
    static constexpr int kWarps = NG == 4 ? 12 : 16;
    static constexpr int kStages = 2;
    static constexpr int kTiles = D == 64 ? 4 : 2;
    static constexpr int kStage = kTiles * Kv4Block<D, NG>::kBytes;
};

// A value that the compiler knows nothing of.
__device__ __forceinline__ void opaque(int& x) { asm volatile("" : "+r"(x)); }

__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x)
{
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / x of a power of two (2^-126 .. 2^126).
__device__ __forceinline__ float inverse_power(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }

// The rest of a wait that has not ended at once (out of line).
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity)
{
    return mbar_wait_bounded(bar, parity, kWaitLimitNs);
}

// Rows whose sums lie in shared memory; those of larger batches in the workspace.
constexpr int kSmemRows = 1024;

// A warp's part of a (row, KV head) that other warps hold parts of, too.
struct PartInfo {
    int32_t b, h;       // b < 0: none
    int32_t begins, ends;
};

__host__ __device__ constexpr int part_floats(int G, int D) { return G * D + ((2 * G + 3) & ~3); }   // o [G][D], m [G], l [G]

template <int D, int NG>
struct AttnSmem {   // byte offsets in dynamic shared memory
    using S = AttnShape<D, NG>;
    static constexpr int R = S::kStages, kRing = R * S::kStage;
    static constexpr int kBars = S::kWarps * kRing;
    static constexpr int kInfo = kBars + S::kWarps * R * 8;
    static constexpr int kHeads = kInfo + S::kWarps * 2 * (int)sizeof(PartInfo);   // a warp's first part: [kWarps][part_floats]
    __host__ __device__ static constexpr int pages(int G) { return kHeads + S::kWarps * part_floats(G, D) * 4; }   // [2][batch + 1]
    __host__ __device__ static constexpr int bytes(int G, int batch) { return pages(G) + (batch <= kSmemRows ? 2 * (batch + 1) * 4 : 0); }
};

// What a lane knows of one tile.
struct Tile {
    const uint8_t* src;   // null: none
    uint32_t bits;        // valid tokens (0 .. 16), kFirst / kLast page of its (row, KV head), which follows
    static constexpr uint32_t kFirst = 32, kLast = 64;
    static __device__ __forceinline__ uint32_t pack(int b, int h) { return (uint32_t)h << 7 | (uint32_t)b << 17; }
    static __device__ __forceinline__ int row(uint32_t bits) { return (int)(bits >> 17); }
    static __device__ __forceinline__ int head(uint32_t bits) { return (int)(bits >> 7 & 1023u); }
};
static_assert(kKv4MaxHeads <= 1024 && kKv4MaxBatch <= 1 << 15, "Tile::pack");

// Sums of o over what lies behind of a (row, KV head), put away every 32 tiles (State::close): in units of
// one, relative to the m of that time.  They lie in the thread's local memory, behind an address
// that the compiler cannot turn into registers: those are full (64 MHA rows 57.9 -> 59.7 us, 8 of 32K tokens
// 40.4 -> 41.6).
template <int D>
struct Closed {
    float4 o[D / 16];
    float m[2];
    __device__ __forceinline__ Closed& hidden()
    {
        Closed* p = this;
        asm volatile("" : "+l"(p) : : "memory");
        return *p;
    }
};

// The running state of a warp for one (row, KV head): lane (g = lane / 4, j =
// lane % 4) holds columns n = 2j and 2j + 1 of everything, tokens g and g + 8 of a
// page's scores, elements 16 mt + g and 16 mt + g + 8 of the output.
template <int D, int NG, class T>
struct State {
    using B = Kv4Block<D, NG>;
    static constexpr int NW = D / 32;     // code words of a lane per 8 tokens
    static constexpr int MT = D / 16;     // 16-element tiles of the output
    // The K accumulators hold 2^-21 q c; sums of q are taken in a unit that the cache's type holds (8 times 2^22 at most).
    static constexpr bool kHalf = std::is_same_v<T, Fp16>;
    static constexpr float kSumUnit = kHalf ? 0x1p-10f : 0x1p-21f;
    uint32_t qf[2 * NW][2];               // q as the K product's column operand
    uint32_t qz[3];                       // (-8, 1) * sum of q over group j, in terms of the cache's type
    float qback[2];                       // undoes q's power of two
    float m[2], l[2];
    float o[MT][4], e[NG][4], z[NG][2];   // e: 15 and 120 times a group's sum p s', in o's unit 2^(E - 24) (apart: a NaN stays in its group)
    float vs[NG][2];                      // 2^-E of each sum: of a group's elements in a column

    bool closed;                          // whether close() has put something away

    __device__ __forceinline__ void start(const AttnArgs& a, int b, int h, int lane)
    {
        const int n = lane >> 2, j = lane & 3;
        uint32_t w[NW][4] = {};
        if (n < a.G) {
            const uint16_t* q = a.q + b * a.q_stride + (int64_t)(h * a.G + n) * D + 8 * j;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const uint4 u = *reinterpret_cast<const uint4*>(q + 32 * i);
                w[i][0] = u.x, w[i][1] = u.y, w[i][2] = u.z, w[i][3] = u.w;
            }
        }
        // The row's largest |q| in the type's own bits, which are in its order.
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) big = __vmaxu2(big, w[i][k] & 0x7fff7fffu);
        big = max(big >> 16, big & 0xffffu);
        big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
        // 2^up takes it into [2^14, 2^15); a row of zeros, or one that is not finite, stays as it is.
        const float top = T::lo(big);
        const int ex = (int)(__float_as_uint(top) >> 23);
        const int up = top == 0.f || ex == 255 ? 0 : max(-126, min(126, 14 + 127 - ex));
        const float mul = __uint_as_float((uint32_t)(127 + up) << 23), back = __uint_as_float((uint32_t)(127 - up) << 23);
        float sums[NG];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // pair k of a word: elements 2k and 2k + 1, at bits 4k; as q meets c * 2^-21, 2^-20, 2^-21, 2^-17
                const float x0 = T::lo(w[i][k]) * mul, x1 = T::hi(w[i][k]) * mul;
                sum += x0 + x1;
                qf[2 * i + (k >> 1)][k & 1] = k & 1 ? pack_f16(x0 * (k == 1 ? 0.5f : 0.0625f), x1 * (k == 1 ? 0.5f : 0.0625f)) : pack_f16(x0, x1);
            }
            sums[i / (NW / NG)] = i % (NW / NG) ? sums[i / (NW / NG)] + sum : sum;
        }
        // Lane j takes its group's sum, in two (fp16) or three (bf16) terms: 22 or 24 bits.
        float rest = 0.f;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], 1);
            sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], 2);
            if (j == k) rest = sums[k] * kSumUnit;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const float term = T::lo(T::pack(rest, 0.f));
            qz[k] = T::pack(-8.f * term, term);
            rest -= term;
        }
        qback[0] = __shfl_sync(0xffffffffu, back, 8 * j);
        qback[1] = __shfl_sync(0xffffffffu, back, 8 * j + 4);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            m[c] = -INFINITY;
            l[c] = 0.f;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[mt][c] = 0.f;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            z[k][0] = z[k][1] = 0.f;
            vs[k][0] = vs[k][1] = 0x1p126f;
#pragma unroll
            for (int c = 0; c < 4; ++c) e[k][c] = 0.f;
        }
        closed = false;
    }

    template <int N>
    static __device__ __forceinline__ void load_shared(uint32_t at, uint32_t (&w)[N])
    {
        if constexpr (N == 4)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
        else if constexpr (N == 2)
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
        else
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(at));
    }

    static __device__ __forceinline__ uint32_t load_shared(uint32_t at)
    {
        uint32_t w[1];
        load_shared(at, w);
        return w[0];
    }

    // The pages of a stage, at `at` in shared memory; `valid`: how many of their
    // tokens count (0 .. 16, a byte for each page; not all none).  Together they
    // share the checks and keep several chains of products in flight.
    static constexpr int NP = AttnShape<D, NG>::kTiles;
    static constexpr int kAll = NP == 4 ? 0x10101010 : 0x1010;
    __device__ __forceinline__ void pages(uint32_t at, int valid, float scale, int lane)
    {
        const int g = lane >> 2;
        int eight = 8;         // a multiplication: the shifts' pipe is the busiest
        opaque(eight);
        const uint32_t codes = at + lane * NW * 4, scales = at + 2 * B::kCodes + g * NG * 4;
        const uint32_t own = scales + (lane & (NG - 1)) * 4;   // group j's word (of lanes that have none: another one's, against zeros)
        float s[NP][4];
        uint32_t mv[NP][2][NG];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            uint32_t ka[NW], kb[NW], mk[2][NG];
            load_shared(codes + p * B::kBytes, ka);
            load_shared(codes + p * B::kBytes + 32 * NW * 4, kb);
            load_shared(scales + p * B::kBytes, mk[0]);
            load_shared(scales + p * B::kBytes + 8 * NG * 4, mk[1]);
            load_shared(scales + p * B::kBytes + B::kScales, mv[p][0]);
            load_shared(scales + p * B::kBytes + B::kScales + 8 * NG * 4, mv[p][1]);
            // sum_groups (z - 8 s) sum q: the scale words (s, z) as they lie against (-8, 1) sum q.
            const float zero[4] = {0.f, 0.f, 0.f, 0.f};
            float base[4];
            uint32_t w0, w1;
            if constexpr (NG == 1) {
                w0 = mk[0][0], w1 = mk[1][0];
            } else {
                w0 = load_shared(own + p * B::kBytes), w1 = load_shared(own + p * B::kBytes + 8 * NG * 4);
            }
            if constexpr (kHalf) {
                mma_f16_16816(base, w0, w1, w0, w1, qz[0], qz[1], zero);
#pragma unroll
                for (int c = 0; c < 4; ++c) base[c] *= 0x1p-21f / kSumUnit;
            } else {
                mma_bf16_16816(base, w0, w1, w0, w1, qz[0], qz[1], zero);
                mma_bf16_16816(base, w0, w1, w0, w1, qz[2], 0u);
            }
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                float acc[4];
#pragma unroll
                for (int i = k * (NW / NG); i < (k + 1) * (NW / NG); ++i) {
                    const uint32_t a0 = ka[i] * eight, b0 = kb[i] * eight, a5 = ka[i] >> 5, b5 = kb[i] >> 5;
                    if (i == k * (NW / NG))
                        mma_f16_16816(acc, a0 & 0x00780078u, b0 & 0x00780078u, ka[i] & 0x00f000f0u, kb[i] & 0x00f000f0u,
                                      qf[2 * i][0], qf[2 * i][1], zero);
                    else
                        mma_f16_16816(acc, a0 & 0x00780078u, b0 & 0x00780078u, ka[i] & 0x00f000f0u, kb[i] & 0x00f000f0u,
                                      qf[2 * i][0], qf[2 * i][1]);
                    mma_f16_16816(acc, a5 & 0x00780078u, b5 & 0x00780078u, a5 & 0x07800780u, b5 & 0x07800780u,
                                  qf[2 * i + 1][0], qf[2 * i + 1][1]);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) base[c] = fmaf(T::lo(mk[c >> 1][k]), acc[c], base[c]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) s[p][c] = base[c];
#pragma unroll
            for (int c = 0; c < 4; ++c) s[p][c] *= scale;   // and by qback where it meets m
        }
        if (valid != kAll) {   // slots past the end may hold anything
#pragma unroll
            for (int p = 0; p < NP; ++p)
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    if (g + 8 * t >= (valid >> (8 * p) & 31)) {
                        s[p][2 * t] = s[p][2 * t + 1] = -INFINITY;
#pragma unroll
                        for (int k = 0; k < NG; ++k) mv[p][t][k] = 0u;
                    }
        }
        // The references m and E move only when a score passes m by more than 4 (log2 units), or a
        // scale 2^(E + 11), or a weight times scale 2^(E + 15): most pages skip the reductions and the rescale.
        float pm[2] = {-INFINITY, -INFINITY}, smax[NG];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            pm[0] = fmaxf(pm[0], fmaxf(s[p][0], s[p][2]));
            pm[1] = fmaxf(pm[1], fmaxf(s[p][1], s[p][3]));
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const float x = fmaxf(fabsf(T::lo(mv[p][0][k])), fabsf(T::lo(mv[p][1][k])));
                smax[k] = p ? fmaxf(smax[k], x) : x;
            }
        }
        pm[0] *= qback[0];
        pm[1] *= qback[1];
        bool moves = pm[0] > m[0] + 4.f || pm[1] > m[1] + 4.f;
#pragma unroll
        for (int k = 0; k < NG; ++k) moves |= smax[k] * fmaxf(vs[k][0], vs[k][1]) > 2048.f;
        if (__any_sync(0xffffffffu, moves)) check_references(pm, smax, s, mv);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float p0 = ex2(fmaf(s[p][0], qback[0], -m[0])), p1 = ex2(fmaf(s[p][1], qback[1], -m[1]));
            const float p2 = ex2(fmaf(s[p][2], qback[0], -m[0])), p3 = ex2(fmaf(s[p][3], qback[1], -m[1]));
            l[0] += p0 + p2;
            l[1] += p1 + p3;
            uint32_t va[NW], vb[NW];
            load_shared(codes + p * B::kBytes + B::kCodes, va);
            load_shared(codes + p * B::kBytes + B::kCodes + 32 * NW * 4, vb);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const float s0 = T::lo(mv[p][0][k]), s1 = T::lo(mv[p][1][k]);
                const float z0 = T::hi(mv[p][0][k]), z1 = T::hi(mv[p][1][k]);
                z[k][0] = fmaf(p0, z0, fmaf(p2, z1, z[k][0]));
                z[k][1] = fmaf(p1, z0, fmaf(p3, z1, z[k][1]));
                // (p s')^T as the column operand: the packed pairs are 8x8 tiles
                // [token][n] in the fragment layout, their transposes are the operand.
                // (In this order: s' 2^-E may pass fp32 where p is 0.)
                const uint32_t b0 = movmatrix_trans(pack_f16(p0 * s0 * vs[k][0], p1 * s0 * vs[k][1]));
                const uint32_t b1 = movmatrix_trans(pack_f16(p2 * s1 * vs[k][0], p3 * s1 * vs[k][1]));
                mma_f16_16816(e[k], 0x000f000fu, 0x00780078u, 0x000f000fu, 0x00780078u, b0, b1);
#pragma unroll
                for (int i = k * (NW / NG); i < (k + 1) * (NW / NG); ++i) {
                    const uint32_t a8 = va[i] >> 8, b8 = vb[i] >> 8;
                    mma_f16_16816(o[2 * i], va[i] & 0x000f000fu, va[i] & 0x00f000f0u, vb[i] & 0x000f000fu, vb[i] & 0x00f000f0u, b0, b1);
                    mma_f16_16816(o[2 * i + 1], a8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x000f000fu, b8 & 0x00f000f0u, b0, b1);
                }
            }
        }
    }

    // What a lane's largest weight and scale make bounds its products: wide scales of small weights may stay.
    __device__ __forceinline__ void check_references(const float (&pm)[2], const float (&smax)[NG], const float (&s)[NP][4], const uint32_t (&mv)[NP][2][NG])
    {
        const float w0 = ex2(pm[0] - m[0]), w1 = ex2(pm[1] - m[1]);   // (NaN where no token of a row counts so far)
        bool moves = w0 > 16.f || w1 > 16.f;
#pragma unroll
        for (int k = 0; k < NG; ++k) moves |= fmaxf(w0 * vs[k][0], w1 * vs[k][1]) * smax[k] > 32768.f;
        if (__any_sync(0xffffffffu, moves)) move_references(pm, s, mv);
    }

    // m follows the lanes' largest scores, E the largest weight times scale.  As m rises, what is in a
    // sum weighs less: E falls with it (rounded up, so that the sum is not made smaller), and then rises to where
    // the tokens at hand are in [2^6, 2^7) if they are above.
    __device__ __forceinline__ void move_references(const float (&pm)[2], const float (&s)[NP][4], const uint32_t (&mv)[NP][2][NG])
    {
        float al[2], fall[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float to = pm[c];
#pragma unroll
            for (int mask = 4; mask < 32; mask <<= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, mask));
            to = fmaxf(to, m[c]);
            const float by = to == m[c] ? 0.f : m[c] - to;   // (at -infinity, too)
            al[c] = ex2(by);
            fall[c] = __uint_as_float((uint32_t)(127 + (int)fminf(ceilf(-by), 100.f)) << 23);
            m[c] = to;
            l[c] *= al[c];
        }
        float top[NG][2];
#pragma unroll
        for (int k = 0; k < NG; ++k) top[k][0] = top[k][1] = 0x1p-120f;   // E >= -126
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float w = ex2(fmaf(s[p][2 * t + c], qback[c], -m[c]));
#pragma unroll
                    for (int k = 0; k < NG; ++k) top[k][c] = fmaxf(top[k][c], fabsf(w * T::lo(mv[p][t][k])));
                }
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            uint32_t most = __byte_perm(__float_as_uint(top[k][0]), __float_as_uint(top[k][1]), 0x7632);   // (exponents are enough)
#pragma unroll
            for (int mask = 4; mask < 32; mask <<= 1) most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, mask));
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float next = __uint_as_float(0x82000000u - ((c ? most : most << 16) & 0x7f800000u));   // 2^6 over the power of two in most
                const float to = fminf(vs[k][c] * fall[c], next), r = to * inverse_power(vs[k][c]) * al[c];
                vs[k][c] = to;
                z[k][c] *= al[c];
                e[k][c] *= r;
                e[k][c + 2] *= r;
#pragma unroll
                for (int mt = k * (MT / NG); mt < (k + 1) * (MT / NG); ++mt) {
                    o[mt][c] *= r;
                    o[mt][c + 2] *= r;
                }
            }
        }
    }

    // o becomes what it stands for, relative to m, with what close() has put away.
    __device__ __forceinline__ void settle(Closed<D>& sums)
    {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int k = mt / (MT / NG);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                o[mt][c] = fmaf(e[k][c], c < 2 ? -8.f / 15.f : -128.f / 120.f, o[mt][c]) * (c < 2 ? 0x1p24f : 0x1p20f) * inverse_power(vs[k][c & 1]);
        }
        if (closed) {
            const Closed<D>& put = sums.hidden();
            const float f0 = put.m[0] == m[0] ? 1.f : ex2(put.m[0] - m[0]), f1 = put.m[1] == m[1] ? 1.f : ex2(put.m[1] - m[1]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const float4 x = put.o[mt];
                o[mt][0] = fmaf(x.x, f0, o[mt][0]);
                o[mt][1] = fmaf(x.y, f1, o[mt][1]);
                o[mt][2] = fmaf(x.z, f0, o[mt][2]);
                o[mt][3] = fmaf(x.w, f1, o[mt][3]);
            }
        }
    }

    // Puts what settle() has made of o away; o and e begin anew (z and l are fp32 sums as it is).
    __device__ __forceinline__ void close(Closed<D>& sums)
    {
        Closed<D>& put = sums.hidden();
        put.m[0] = m[0];
        put.m[1] = m[1];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            put.o[mt] = make_float4(o[mt][0], o[mt][1], o[mt][2], o[mt][3]);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[mt][c] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < NG; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c) e[k][c] = 0.f;
        closed = true;
    }

    // The sums over all lanes' tokens; o (settled) is then the unnormalised output.
    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int mask = 4; mask < 32; mask <<= 1) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                l[c] += __shfl_xor_sync(0xffffffffu, l[c], mask);
#pragma unroll
                for (int k = 0; k < NG; ++k) z[k][c] += __shfl_xor_sync(0xffffffffu, z[k][c], mask);
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[mt][c] += z[mt / (MT / NG)][c & 1];
    }

    __device__ __forceinline__ void write_out(const AttnArgs& a, int b, int h, int lane) const
    {
        const int g = lane >> 2;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int n = 2 * (lane & 3) + c;
            if (n >= a.G) continue;
            const float inv = l[c] == 0.f ? 0.f : rcp(l[c]);
            uint16_t* out = a.out + b * a.out_stride + (int64_t)(h * a.G + n) * D + g;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const uint32_t w = T::pack_finite(o[mt][c] * inv, o[mt][c + 2] * inv);
                out[16 * mt] = (uint16_t)w;
                out[16 * mt + 8] = (uint16_t)(w >> 16);
            }
            if (a.lse && g == 0) a.lse[(int64_t)b * a.Hq + h * a.G + n] = (m[c] + lg2(l[c])) * kLn2;
        }
    }

    __device__ __forceinline__ void write_part(float* part, int G, int lane) const
    {
        const int g = lane >> 2;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int n = 2 * (lane & 3) + c;
            if (n >= G) continue;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                part[n * D + 16 * mt + g] = o[mt][c];
                part[n * D + 16 * mt + 8 + g] = o[mt][c + 2];
            }
            if (g == 0) {
                part[G * D + n] = m[c];
                part[G * (D + 1) + n] = l[c];
            }
        }
    }
};

// One query row of merged parts: o elements lane * E .. of this lane, m and l.
template <int D>
struct RowSum {
    static constexpr int E = D / 32;
    float o[E], m, l;
    __device__ __forceinline__ RowSum() : m(-INFINITY), l(0.f)
    {
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = 0.f;
    }
    // Adds row n of the first `count` lanes' parts, in the lanes' order: `at` is a
    // part's offset in floats from `base` (shared memory, or global memory, whose L1 is
    // passed by), -1 for none (not the first lane's).  A lane loads its part's (m, l),
    // all lanes the rows, U in flight, the first ones before the weights are known.
    template <int U, bool kGlobal>
    __device__ __forceinline__ void merge(const float* base, int at, int count, int G, int n, int lane)
    {
        const bool mine = lane < count && at >= 0;
        const int other = __shfl_sync(0xffffffffu, at, 0), from = mine ? at : other;   // something to load where there is nothing to add
        float mc = load<kGlobal>(base + from + G * D + n), lc = load<kGlobal>(base + from + G * (D + 1) + n);
        if (!mine) {
            mc = -INFINITY;
            lc = 0.f;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, mine);
        float w = 0.f;
#pragma unroll 1
        for (int c = 0; c < count; c += U) {
            float x[U][E];
#pragma unroll
            for (int u = 0; u < U; ++u) load<kGlobal>(base + __shfl_sync(0xffffffffu, from, (c + u) & 31) + n * D + lane * E, x[u]);
            if (c == 0) {
                const float top = fmaxf(m, warp_max(mc)), al = m == top ? 1.f : ex2(m - top);
                w = !mine ? 0.f : mc == top ? 1.f : ex2(mc - top);
                lc *= w;
                m = top;
                l *= al;
#pragma unroll
                for (int i = 0; i < E; ++i) o[i] *= al;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool on = c + u < 32 && ((some >> (c + u)) & 1u);
                const float wu = __shfl_sync(0xffffffffu, w, (c + u) & 31), lu = __shfl_sync(0xffffffffu, lc, (c + u) & 31);
                l += on ? lu : 0.f;
#pragma unroll
                for (int i = 0; i < E; ++i) o[i] = fmaf(on ? x[u][i] : 0.f, wu, o[i]);
            }
        }
    }
    static __device__ __forceinline__ float warp_max(float x)   // (a NaN only where all are)
    {
        float y;
        asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
        return y;
    }
    __device__ __forceinline__ void write_part(float* part, int G, int n, int lane) const
    {
        if constexpr (E == 4) *reinterpret_cast<float4*>(part + n * D + lane * 4) = make_float4(o[0], o[1], o[2], o[3]);
        else *reinterpret_cast<float2*>(part + n * D + lane * 2) = make_float2(o[0], o[1]);
        if (lane == 0) {
            part[G * D + n] = m;
            part[G * (D + 1) + n] = l;
        }
    }
    template <bool kGlobal>
    static __device__ __forceinline__ float load(const float* p)
    {
        if constexpr (kGlobal) return __ldcg(p);
        return *p;
    }
    template <bool kGlobal>
    static __device__ __forceinline__ void load(const float* p, float (&x)[E])
    {
        if constexpr (E == 4) {
            const float4 v = kGlobal ? __ldcg(reinterpret_cast<const float4*>(p)) : *reinterpret_cast<const float4*>(p);
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        } else {
            const float2 v = kGlobal ? __ldcg(reinterpret_cast<const float2*>(p)) : *reinterpret_cast<const float2*>(p);
            x[0] = v.x, x[1] = v.y;
        }
    }
    template <class T>
    __device__ __forceinline__ void write_out(const AttnArgs& a, int b, int h, int n, int lane) const
    {
        const float inv = l == 0.f ? 0.f : rcp(l);
        uint16_t* out = a.out + b * a.out_stride + (int64_t)(h * a.G + n) * D + lane * E;
#pragma unroll
        for (int i = 0; i < E; i += 2) *reinterpret_cast<uint32_t*>(out + i) = T::pack_finite(o[i] * inv, o[i + 1] * inv);
        if (a.lse && lane == 0) a.lse[(int64_t)b * a.Hq + h * a.G + n] = (m + lg2(l)) * kLn2;
    }
};

// x / H for a multiple x of H.
__device__ __forceinline__ uint32_t multiple_over(uint32_t x, uint32_t H, uint32_t H_inv)
{
    const uint32_t q = __umulhi(x, H_inv);
    return q + (x - q * H >= H);
}

// The warps' shares: the first `extra` of them have base + 1 places, the others base; the warps of a CTA that have one.
struct Shares {
    uint32_t base, extra, cta_warps;
};

// What is left when the CTA's warps have worked their shares: rows without
// tokens, the merges of what lies in this CTA, the span of what goes on after it.  (Out of line: the
// registers that this takes are not the main loop's.)
template <int D, int NG, class T>
__device__ __noinline__ void finish_cta(const AttnArgs& a, uint8_t* smem, const Shares sh, bool all_held)
{
    using S = AttnShape<D, NG>;
    using M = AttnSmem<D, NG>;
    constexpr int W = S::kWarps;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t H = a.H;
    const PartInfo* infos = reinterpret_cast<const PartInfo*>(smem + M::kInfo);
    const uint32_t* pages = a.batch <= kSmemRows ? reinterpret_cast<const uint32_t*>(smem + M::pages(a.G)) : a.sums;
    const uint32_t* costs = pages + a.batch + 1;
    // Rows without tokens.
    if (!all_held)
#pragma unroll 1
        for (int r = blockIdx.x; r < a.batch; r += gridDim.x)
            if (pages[r] == pages[r + 1]) {
#pragma unroll 1
                for (int i = tid; i < a.Hq * (D / 8); i += W * 32)
                    *reinterpret_cast<uint4*>(a.out + r * a.out_stride + i * 8) = make_uint4(0u, 0u, 0u, 0u);
                if (a.lse)
#pragma unroll 1
                    for (int i = tid; i < a.Hq; i += W * 32) a.lse[(int64_t)r * a.Hq + i] = -INFINITY;
            }
    __syncthreads();

    // This CTA's parts, in the order of the list, one in each lane: a group of
    // them belongs to one (row, KV head).
    const int PF = part_floats(a.G, D);
    const PartInfo mine = lane < 2 * W ? infos[lane] : PartInfo{-1, 0, 0, 0};
    const uint32_t valid = __ballot_sync(0xffffffffu, mine.b >= 0);
    const uint32_t begin = __ballot_sync(0xffffffffu, mine.b >= 0 && mine.begins);
    const uint32_t ending = __ballot_sync(0xffffffffu, mine.b >= 0 && mine.ends);
    const uint32_t groups = begin | (valid & (0u - valid));
    if (warp == W - 1 && lane == 0) {
        PartSpan span{-1, 0, 0, 0};
        const int last = 31 - __clz(groups);   // (the last group begins here, or it is the only one)
        if (begin && !(ending >> last) && ((begin >> last) & 1u)) {
            // It goes on: the CTA whose share holds its last page.
            const PartInfo in = infos[last];
            const uint32_t n = multiple_over(pages[in.b + 1] - pages[in.b], H, a.H_inv);
            const uint32_t place = costs[in.b] + (in.h + 1) * (n + kRowCost) - 1, long_ones = sh.extra * (sh.base + 1);
            const bool in_long = place < long_ones;
            const uint32_t w = (in_long ? place : place - long_ones) / (in_long ? sh.base + 1 : sh.base) + (in_long ? 0 : sh.extra);
            span = {in.b, in.h, (int)(w / sh.cta_warps), 0};
        }
        a.spans[blockIdx.x] = span;
    }
    const int jobs = __popc(groups) * a.G;
#pragma unroll 1
    for (int job = warp; job < jobs; job += W) {
        uint32_t rest = groups;
        const int group = (int)(job * a.G_inv >> 16), n = job - group * a.G;   // job / G
#pragma unroll 1
        for (int u = group; u > 0; --u) rest &= rest - 1u;
        const int e = __ffs(rest) - 1, i = e + lane;
        rest &= rest - 1u;
        const uint32_t members = valid & (0xffffffffu << e) & (rest ? (rest & (0u - rest)) - 1u : 0xffffffffu);
        const PartInfo row = infos[e];
        RowSum<D> sum;
        const int off = i > 31 || !((members >> i) & 1u) ? -1 : i & 1 ? (i >> 1) * (M::kRing / 4) : M::kHeads / 4 + (i >> 1) * PF;
        sum.template merge<4, false>(reinterpret_cast<const float*>(smem), off, 32 - __clz(members) - e, a.G, n, lane);
        if (row.begins && (ending & members)) sum.template write_out<T>(a, row.b, row.h, n, lane);
        else sum.write_part(a.parts + ((int64_t)blockIdx.x * 2 + row.begins) * PF, a.G, n, lane);
    }
}

template <int D, int NG, class T>
__global__ void __launch_bounds__(AttnShape<D, NG>::kWarps * 32, 1) attention_kernel(const __grid_constant__ AttnArgs a)
{
    using S = AttnShape<D, NG>;
    using B = Kv4Block<D, NG>;
    using M = AttnSmem<D, NG>;
    constexpr int W = S::kWarps, N = S::kTiles, R = S::kStages;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint2 warp_pages[W];
    static_assert(2 * W <= 32, "a lane for each part");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* ring = smem + warp * M::kRing;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + M::kBars) + warp * R;
    PartInfo* infos = reinterpret_cast<PartInfo*>(smem + M::kInfo);
    float* heads = reinterpret_cast<float*>(smem + M::kHeads);
    // Tiles of the rows before each row, and the same with kRowCost for each (row, KV head) that has some.
    uint32_t* pages = a.batch <= kSmemRows ? reinterpret_cast<uint32_t*>(smem + M::pages(a.G)) : a.sums;
    uint32_t* costs = pages + a.batch + 1;
    if (lane < R) mbar_init(smem_addr(bars + lane), 1);
    fence_mbar_init();
    if (tid < 2 * W) infos[tid].b = -1;
    griddep_wait();
    griddep_launch_dependents();

    // Pages of the rows before each row.
    const uint32_t H = a.H;
    int has_ids = a.seq_ids != nullptr;
    opaque(has_ids);
    const int max_len = min(a.max_pages, (1 << 27) - 1) * kPageSize;
    if (tid == 0) pages[0] = costs[0] = 0;
    uint64_t all_pages = 0;
    uint32_t held = 0;        // rows that are not empty
#pragma unroll 1
    for (int r0 = 0; r0 < a.batch; r0 += W * 32) {
        const int r = r0 + tid;
        uint32_t n = 0;
        if (r < a.batch) {
            const int seq = has_ids ? a.seq_ids[r] : r;
            int len = seq >= 0 && seq < a.max_seqs ? a.lens[seq] : -1;
            if (len < 0 || len > max_len) {
                if (blockIdx.x == 0) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
                len = 0;
            }
            n = (uint32_t)(len + kPageSize - 1) / kPageSize;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, n != 0);
        uint32_t sum = n;     // (below 2^32: rows have less than 2^27 pages)
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, sum, k);
            if (lane >= k) sum += up;
        }
        if (lane == 31) warp_pages[warp] = make_uint2(sum, (uint32_t)__popc(some));
        __syncthreads();
        // The same over the warps (a lane for each); the total in 64 bits.
        const uint2 of = lane < W ? warp_pages[lane] : make_uint2(0u, 0u);
        const uint32_t mine = (uint32_t)all_pages + __reduce_add_sync(0xffffffffu, lane < warp ? of.x : 0u);
        uint32_t rows = held + __reduce_add_sync(0xffffffffu, lane < warp ? of.y : 0u);
        all_pages += __reduce_add_sync(0xffffffffu, of.x & 0xffffu) + ((uint64_t)__reduce_add_sync(0xffffffffu, of.x >> 16) << 16);
        held += __reduce_add_sync(0xffffffffu, of.y);
        if (r < a.batch) {
            const uint32_t up_to = mine + sum;
            rows += __popc(some & (2u << lane) - 1u);
            pages[r + 1] = up_to * H;
            costs[r + 1] = (up_to + rows * kRowCost) * H;
        }
        if (r0 + W * 32 < a.batch) __syncthreads();
    }
    __syncthreads();
    if (all_pages * a.H > 0x7fffffffull) {   // the same in all threads
        if (tid == 0) a.spans[blockIdx.x] = {-1, 0, 0, 0};
        if (blockIdx.x == 0 && tid == 0) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
        return;
    }

    // Shares: equal parts of the list of tiles in which every (row, KV head)
    // is preceded by kRowCost empty places; the first `extra` warps take one place more.
    const uint32_t places = costs[a.batch];
    const uint32_t wanted = (places + kMinShare - 1) / kMinShare;
    const uint32_t cta_warps = min((uint32_t)W, max(kMinWarps, (wanted + gridDim.x - 1) / gridDim.x));   // that work, of each CTA
    const uint32_t warps = min(gridDim.x * cta_warps, wanted);
    const uint32_t base = warps ? places / warps : 0, extra = warps ? places % warps : 0;
    // The last row from r0 on with sums[row] <= x (so not empty, where x < sums[batch]); sums[r0] <= x.
    auto row_of = [&](const uint32_t* sums, int r0, uint32_t x) {
        int step = 1;
#pragma unroll 1
        for (; r0 + step < a.batch && sums[r0 + step] <= x; step *= 2) r0 += step;
        int r1 = min(r0 + step, a.batch);
#pragma unroll 1
        while (r1 - r0 > 1) {
            const int mid = (r0 + r1) >> 1;
            if (sums[mid] <= x) r0 = mid;
            else r1 = mid;
        }
        return r0;
    };
    auto over_H = [&](uint32_t x) { return multiple_over(x, H, a.H_inv); };
    auto head_of = [&](uint32_t x, uint32_t n) {   // x / n, below 1024
        int q = (int)__fdividef((float)x, (float)n);
        q -= q * (int64_t)n > x;
        return (uint32_t)(q + (x - q * n >= n));
    };
    uint32_t lo = 0;
    int row0 = 0;             // the row that this lane's next tile is at or behind
    {   // lane 0: tiles before this warp's share, lane 1: up to its end
        const uint32_t w = min(blockIdx.x * cta_warps + min((uint32_t)warp + (lane & 1), cta_warps), warps), at = w * base + min(w, extra);
        if (w < warps) {
            const int r = row_of(costs, 0, at);
            const uint32_t n = over_H(costs[r + 1] - costs[r]), in_row = at - costs[r], h = head_of(in_row, n), off = in_row - h * n;
            row0 = r;
            lo = pages[r] + h * (n - kRowCost) + (off > kRowCost ? off - kRowCost : 0);
        } else {
            lo = pages[a.batch];
        }
    }
    const int count = (int)(__shfl_sync(0xffffffffu, lo, 1) - __shfl_sync(0xffffffffu, lo, 0));
    lo = __shfl_sync(0xffffffffu, lo, 0);
    row0 = __shfl_sync(0xffffffffu, row0, 0);
    const uint64_t policy = l2_policy_evict_first();

    bool ok = true;
    auto tile_of = [&](int i) {   // tile i of this warp's share
        Tile t{nullptr, 0};
        if (i >= count || !ok) return t;
        const uint32_t at = lo + i;
        const int r0 = row0 = row_of(pages, row0, at);
        const uint32_t n = over_H(pages[r0 + 1] - pages[r0]), in_row = at - pages[r0];
        const int h = (int)head_of(in_row, n), p = (int)(in_row - h * n);
        const int seq = has_ids ? a.seq_ids[r0] : r0;
        const int32_t page = a.block_table[(int64_t)seq * a.max_pages + p];
        int valid = min(kPageSize, a.lens[seq] - p * kPageSize);
        if (page >= 0 && page < a.num_pages) {
            t.src = a.pool + ((int64_t)page * a.H + h) * B::kBytes;
        } else {                      // read page 0 in its place, and leave its tokens out
            kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
            t.src = a.pool;
            valid = 0;
        }
        t.bits = Tile::pack(r0, h) | valid | (p == 0 ? Tile::kFirst : 0u) | (p == (int)n - 1 ? Tile::kLast : 0u);
        return t;
    };
    // The ring's stages hold N tiles each and are used in turn: tiles N k .. of
    // the share lie in stage k % R.  Their copies are started by the lanes that hold the tiles.
    const uint32_t ring_at = smem_addr(ring), bars_at = smem_addr(bars);
    const uint32_t ring_lane = ring_at + (lane % N) * B::kBytes;

    State<D, NG, T> st;
    Closed<D> closed_sums;
    Tile next{nullptr, 0};            // of the 32 tiles after those in work
    const uint8_t* from = nullptr;    // the tile that this lane starts next, in turn `when` of the 32 / N (-1: none),
    int when = -1;
    uint32_t expect = 0;              // and the bytes that it announces: of its stage's tiles
    auto take_next = [&](int i) {     // the copies of `next`, whose first tile is i
        from = next.src;
        when = from ? lane / N : -1;
        expect = from && lane % N == 0 ? min(N, count - i - lane) * B::kBytes : 0u;
    };
    uint32_t cur = 0;                 // of a tile in work: Tile::bits
    constexpr uint32_t kOpen = 1, kClose = 2, kRefill = 4, kFull = 8, kHold = 16;   // and from bit 8 on, if not kFull: tiles
    uint32_t what = kRefill;          // and what the turn that begins with it has to do
    int at = -32;                     // the tile that the next refill begins with
    bool begins = true;
    uint32_t stage = 0;               // stages done, from the share's first on
#pragma unroll 1
    for (int i = 0; i < count;) {
        const int src = i & 31;
        uint32_t turn = __shfl_sync(0xffffffffu, what, src);
        int valid = State<D, NG, T>::kAll, tiles = N;
        if (turn != kFull) {          // not just a stage of full pages
            if (turn & kRefill) {
                cur = next.bits;
                next = tile_of(at + 32 + lane);
                if (at < 0) {         // fill the ring
                    take_next(0);
                    __syncwarp();
                    bulk_load_turn(ring_lane + lane / N * S::kStage, from, B::kBytes, expect, bars_at + 8 * (lane / N), policy, when,
                                   lane < N * R ? lane / N : -2);
                    at = 0;
                    continue;
                }
                at += 32;
                // A turn takes a stage's tiles as far as they are pages of one row.
                const uint32_t lasts = __ballot_sync(0xffffffffu, cur & Tile::kLast);
                const uint32_t fulls = __ballot_sync(0xffffffffu, (cur & 31) == kPageSize);
                const uint32_t closes = lasts | (i + 32 < count ? 0u : 1u << (count - 1 - i));
                constexpr uint32_t kEnds = N == 4 ? 0x88888888u : 0xaaaaaaaau;   // a stage's last tile
                const int run = __ffs((closes | kEnds) >> lane);
                const bool full = run == N && (~fulls >> lane & ((1u << N) - 1u)) == 0;
                what = ((cur & Tile::kFirst) || i + lane == 0 ? kOpen : 0u) | (closes >> (lane + run - 1) & 1u ? kClose : 0u) |
                       (lane == 0 ? kRefill : 0u) | (kEnds >> (lane + run - 1) & 1u ? 0u : kHold) | (full ? kFull : (uint32_t)run << 8);
                turn = __shfl_sync(0xffffffffu, what, 0);
            }
            if (turn & kOpen) {       // before the wait: q arrives meanwhile
                const uint32_t t = __shfl_sync(0xffffffffu, cur, src);
                begins = t & Tile::kFirst;
                st.start(a, Tile::row(t), Tile::head(t), lane);
            }
            if (!(turn & kFull)) {
                tiles = (int)(turn >> 8);
                valid = 0;
#pragma unroll
                for (int p = 0; p < N; ++p) {
                    const int t = (src & ~(N - 1)) + p, v = (int)(__shfl_sync(0xffffffffu, cur, t) & 31);
                    if (t >= src && t < src + tiles) valid |= v << (8 * p);
                }
            }
        }
        const uint32_t place = stage % R, bar = bars_at + 8 * place, parity = stage / R & 1u;
        if (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)) && ok) {
            ok = __all_sync(0xffffffffu, wait_long(bar, parity));
            if (!ok) {   // no more copies; those in flight land first, and the result is void
                if (lane == 0) kv4_error(a.err, KVC_DEVERR_WAIT_TIMEOUT);
#pragma unroll 1
                for (int k = i / N; k < min(i / N + R, (count + N - 1) / N); ++k) wait_long(bars_at + 8 * (k % R), (k / R) & 1);
                when = -1;
                next.src = nullptr;
            }
        }
        opaque(valid);                // (one copy of the work, not one for each kind of turn: code is fetched once a launch)
        if (valid) st.pages(ring_at + place * S::kStage, valid, a.scale, lane);
        i += tiles;
        if ((turn & (kClose | kHold)) || (i & 31) == 0) {
            if ((turn & kClose) || (i & 31) == 0) st.settle(closed_sums);   // (one copy of it)
            if (!(turn & (kClose | kHold))) st.close(closed_sums);
            if (turn & kClose) {
                const uint32_t t = __shfl_sync(0xffffffffu, cur, (i - 1) & 31);
                const int b = Tile::row(t), h = Tile::head(t);
                const bool ends = t & Tile::kLast;
                st.finish();
                if (begins && ends) {
                    st.write_out(a, b, h, lane);
                } else {
                    // A part that is not the share's last one began before it.
                    const int k = i == count ? 1 : 0;
                    __syncwarp();     // the ring's last tiles have been read
                    st.write_part(k ? reinterpret_cast<float*>(ring) : heads + warp * part_floats(a.G, D), a.G, lane);
                    if (lane == 0) infos[2 * warp + k] = {b, h, begins, ends};
                }
            }
            if (turn & kHold) continue;   // more of the stage is to come
        }
        __syncwarp();
        const int issue = (stage + R) & (32 / N - 1);
        if (issue == 0) take_next((stage + R) * N);
        bulk_load_turn(ring_lane + place * S::kStage, from, B::kBytes, expect, bar, policy, when, issue);
        ++stage;
    }

    finish_cta<D, NG, T>(a, smem, Shares{base, extra, cta_warps}, (int)held == a.batch);
}

// What crosses CTAs: a warp merges one query row of the (row, KV head) that
// goes on after some CTA of the launch before this one.
constexpr int kMergeWarps = 8;
template <int D, class T>
__global__ void __launch_bounds__(kMergeWarps * 32) merge_kernel(const __grid_constant__ AttnArgs a, int ctas)
{
    const int lane = threadIdx.x & 31, w = blockIdx.x * kMergeWarps + (threadIdx.x >> 5);
    const int c = (int)(w * a.G_inv >> 16), n = w - c * a.G, PF = part_floats(a.G, D);   // w / G
    griddep_wait();
    griddep_launch_dependents();
    if (c >= ctas) return;
    const PartSpan span = a.spans[c];
    if (span.b < 0) return;
    const int parts = span.last - c + 1;
    RowSum<D> sum;
#pragma unroll 1
    for (int i0 = 0; i0 < parts; i0 += 32) {
        const int i = i0 + lane;
        sum.template merge<8, true>(a.parts, ((c + i) * 2 + (i == 0 ? 1 : 0)) * PF, min(32, parts - i0), a.G, n, lane);
    }
    sum.template write_out<T>(a, span.b, span.h, n, lane);
}

int device_sms()
{
    static std::atomic<int> known[OncePerDevice::kDevices] = {};
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    if (dev < OncePerDevice::kDevices && (n = known[dev].load(std::memory_order_relaxed))) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev < OncePerDevice::kDevices) known[dev].store(n, std::memory_order_relaxed);
    return n;
}

// The workspace: spans, sums of large batches, parts.
struct Workspace {
    int64_t sums, parts, bytes;   // offsets of the latter two, and the whole
    Workspace(int sms, int G, int D)
    {
        sums = 256 * ((sms * (int64_t)sizeof(PartSpan) + 255) / 256);
        parts = sums + 256 * ((2 * (kKv4MaxBatch + 1) * 4 + 255) / 256);
        bytes = parts + (int64_t)sms * 2 * part_floats(G, D) * 4;
    }
};

struct LaunchAttention {
    AttnArgs& a;
    int sms;
    cudaStream_t st;
    template <int D, int NG, class T>
    cudaError_t operator()() const
    {
        using S = AttnShape<D, NG>;
        using M = AttnSmem<D, NG>;
        constexpr int kMost = M::bytes(kMaxGroup, kSmemRows);
        static_assert(part_floats(kMaxGroup, D) * 4 <= M::kRing, "a part lies in its warp's ring");
        static_assert(kMost <= 226 * 1024, "shared memory of a CTA, beside its static part");
        static OncePerDevice once;
        if (cudaError_t e = once.set_attribute(attention_kernel<D, NG, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost); e != cudaSuccess)
            return e;
        cudaError_t e = kv4_launch(attention_kernel<D, NG, T>, dim3((unsigned)sms), S::kWarps * 32, (size_t)M::bytes(a.G, a.batch), st, a);
        if (e == cudaSuccess)
            e = kv4_launch(merge_kernel<D, T>, dim3((unsigned)((sms * a.G + kMergeWarps - 1) / kMergeWarps)), kMergeWarps * 32, 0, st, a, sms);
        return e;
    }
};

int check_heads(const kv4_pool* pool, int32_t num_q_heads) noexcept
{
    if (num_q_heads < 1 || num_q_heads % pool->num_kv_heads)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: num_q_heads must be a positive multiple of num_kv_heads");
    if (num_q_heads / pool->num_kv_heads > kMaxGroup)
        return kv4_fail(KVC_ERR_UNSUPPORTED, "kv4_decode_attention: more than 8 query heads per KV head");
    return KVC_OK;
}

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int64_t kv4_workspace_bytes(const kv4_pool* pool, int32_t num_q_heads)
{
    if (int rc = kv4_check_pool(pool, false)) return rc;
    if (int rc = check_heads(pool, num_q_heads)) return rc;
    const int sms = device_sms();
    if (!sms) return kv4_fail(KVC_ERR_CUDA, "kv4_workspace_bytes: cannot query the current device");
    return Workspace(sms, num_q_heads / pool->num_kv_heads, pool->head_dim).bytes;
}

extern "C" KVC_API int kv4_decode_attention(const kv4_pool* pool, const kv_tables* tables, int32_t batch,
                                            const int32_t* seq_ids, int32_t num_q_heads, const void* q, int64_t q_stride,
                                            void* out, int64_t out_stride, float* lse, float softmax_scale,
                                            void* workspace, int64_t workspace_bytes, int32_t* device_error, void* stream)
{
    if (int rc = kv4_check_pool(pool, true)) return rc;
    if (int rc = kv4_check_tables(tables)) return rc;
    if (int rc = check_heads(pool, num_q_heads)) return rc;
    if (batch < 1 || batch > kKv4MaxBatch) return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: batch must be in 1 .. 4096");
    if (!seq_ids && batch > tables->max_seqs)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: more rows than requests, and no seq_ids");
    if (!q || !out || !workspace) return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: null argument");
    if (!kv4_aligned(q, 16) || !kv4_aligned(out, 16) || q_stride % 8 || out_stride % 8)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: rows must be 16-byte aligned, strides multiples of 8 elements");
    if (batch > 1 && (q_stride < 0 || out_stride < (int64_t)num_q_heads * pool->head_dim))
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: q_stride must be >= 0, out rows must not overlap");
    if (!(softmax_scale < 0x1p100f))   // (with the scores' unit it has to be a number of 32 bits)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: softmax_scale must be below 2^100");
    if (!kv4_aligned(workspace, 256) || workspace_bytes < 256)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: workspace must be 256-byte aligned and of kv4_workspace_bytes()");
    const int sms = device_sms();
    if (!sms) return kv4_fail(KVC_ERR_CUDA, "kv4_decode_attention: cannot query the current device");
    const int G = num_q_heads / pool->num_kv_heads;
    const Workspace ws(sms, G, pool->head_dim);
    if (workspace_bytes < ws.bytes)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: the workspace is smaller than kv4_workspace_bytes()");
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)pool->head_dim);
    AttnArgs a{};
    a.pool = static_cast<const uint8_t*>(pool->data);
    a.num_pages = pool->num_pages;
    a.H = pool->num_kv_heads;
    a.H_inv = a.H == 1 ? 0xffffffffu : (uint32_t)(((uint64_t)1 << 32) / a.H);
    a.G_inv = (uint32_t)((65536 + G - 1) / G);
    a.Hq = num_q_heads;
    a.G = G;
    a.block_table = tables->block_table;
    a.lens = tables->lens;
    a.max_seqs = tables->max_seqs;
    a.max_pages = tables->max_pages;
    a.batch = batch;
    a.seq_ids = seq_ids;
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.lse = lse;
    a.scale = scale * 1.4426950408889634f * 0x1p21f;
    a.err = device_error;
    uint8_t* const work = static_cast<uint8_t*>(workspace);
    a.spans = reinterpret_cast<PartSpan*>(work);
    a.sums = reinterpret_cast<uint32_t*>(work + ws.sums);
    a.parts = reinterpret_cast<float*>(work + ws.parts);
    return kv4_launch_result(kv4_dispatch(*pool, LaunchAttention{a, sms, static_cast<cudaStream_t>(stream)}));
}
