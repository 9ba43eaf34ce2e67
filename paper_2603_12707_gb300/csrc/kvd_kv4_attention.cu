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
// subnormal, c * 2^-24 in bits 0-3 and c * 2^-20 in bits 4-7, whose product with
// another fp16 is exact.  Eight codes take five instructions to become four
// operands.  The other operand is q, scaled by a power of two into fp16's range
// (divided by 16 where it meets bits 4-7), or p * s', relative to a power of
// two 2^E that follows the largest s'.  The 8 is subtracted by starting QK's
// accumulators at -8 sum q, and for PV by one more product with rows of -8 (so
// that p * s' is rounded once for both).
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
// it holds; what crosses CTAs goes through the workspace and the last CTA to
// arrive (a counter per first CTA, which it sets back to zero) merges the parts in
// the order of the list.
#include <cmath>

#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr uint64_t kWaitLimitNs = 1000000000ull;
constexpr float kLn2 = 0.6931471805599453f;
// What starting and ending a (row, KV head) costs a warp, in tiles: shares count it.
constexpr uint32_t kRowCost = 3;
// What a warp takes at least, in tiles: a small call uses fewer warps rather than merge more parts.
constexpr uint32_t kMinShare = 2;

constexpr int kCtasPerSm = 2;

struct AttnArgs {
    const uint8_t* pool;
    int64_t num_pages;
    int32_t H, Hq, G;
    const int32_t* block_table;
    const int32_t* lens;
    int32_t max_seqs, max_pages, batch;
    const int32_t* seq_ids;
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    float* lse;
    float scale;         // softmax scale * log2(e) * 2^24 (the accumulators' unit)
    int32_t* counters;   // [grid]: CTAs that have left their part of the row that starts in CTA i; zero between calls
    float* parts;        // [grid][2][G][D + 2]: a CTA's part of the row that began before it, and of the one that goes on
    int32_t* err;
};

// The shape of a variant: warps per CTA, CTAs per SM, ring stages (of two tiles) per warp.
template <int D, int NG>
struct AttnShape {
    static constexpr int kWarps = NG == 4 ? 6 : 8;
    static constexpr int kCtas = kCtasPerSm;
    static constexpr int kStages = D == 64 ? 4 : 2;
    static constexpr int kRing = kStages * 2 * Kv4Block<D, NG>::kBytes;   // of one warp
};

// The rest of a wait that has not ended at once (out of line).
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity)
{
    return mbar_wait_bounded(bar, parity, kWaitLimitNs);
}

// A warp's part of a (row, KV head) that other warps hold parts of, too.
struct PartInfo {
    int32_t b, h;       // b < 0: none
    int32_t begins, ends;
};

__host__ __device__ constexpr int part_floats(int G, int D) { return G * (D + 2); }   // o [G][D], m [G], l [G]

template <int D, int NG>
struct AttnSmem {   // byte offsets in dynamic shared memory
    using S = AttnShape<D, NG>;
    static constexpr int kBars = S::kWarps * S::kRing;
    static constexpr int kInfo = kBars + S::kWarps * S::kStages * 8;
    static constexpr int kHeads = kInfo + S::kWarps * 2 * (int)sizeof(PartInfo);   // a warp's first part: [kWarps][part_floats]
    __host__ __device__ static constexpr int pages(int G) { return kHeads + S::kWarps * part_floats(G, D) * 4; }   // [batch + 1]
    __host__ __device__ static constexpr int costs(int G, int batch) { return pages(G) + (batch + 1) * 4; }        // [batch + 1]
    __host__ __device__ static constexpr int last(int G, int batch) { return costs(G, batch) + (batch + 1) * 4; }  // [batch] bytes
    __host__ __device__ static constexpr int bytes(int G, int batch) { return last(G, batch) + batch; }
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

// The running state of a warp for one (row, KV head): lane (g = lane / 4, j =
// lane % 4) holds columns n = 2j and 2j + 1 of everything, tokens g and g + 8 of a
// page's scores, elements 16 mt + g and 16 mt + g + 8 of the output.
template <int D, int NG, class T>
struct State {
    using B = Kv4Block<D, NG>;
    static constexpr int NW = D / 32;     // code words of a lane per 8 tokens
    static constexpr int MT = D / 16;     // 16-element tiles of the output
    uint32_t qf[2 * NW][2];               // q as the K product's column operand
    float qsum[NG][2];                    // sum of q over a group, in the accumulators' units
    float qoff[4];                        // -8 times it, as the accumulators begin (kept for one group: registers)
    float qback[2];                       // undoes q's power of two
    float m[2], l[2];
    float o[MT][4], e[NG][4], z[NG][2];
    float vs, vlimit;                     // 2^-E, and the scale above which E moves

    __device__ __forceinline__ void start(const AttnArgs& a, int b, int h, int lane)
    {
        const int n = lane >> 2, j = lane & 3;
        uint4 w[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (n < a.G)
                w[i] = *reinterpret_cast<const uint4*>(a.q + b * a.q_stride + (int64_t)(h * a.G + n) * D + 32 * i + 8 * j);
        }
        float x[NW][8], top = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[i][2 * k] = T::lo(u[k]);
                x[i][2 * k + 1] = T::hi(u[k]);
                top = fmaxf(top, fmaxf(fabsf(x[i][2 * k]), fabsf(x[i][2 * k + 1])));
            }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^up takes the row's largest |q| into [2^14, 2^15); a row of zeros, or one that is not finite, stays as it is.
        const int ex = (int)(__float_as_uint(top) >> 23);
        const int up = top == 0.f || ex == 255 ? 0 : max(-126, min(126, 14 + 127 - ex));
        const float mul = __uint_as_float((uint32_t)(127 + up) << 23), back = __uint_as_float((uint32_t)(127 - up) << 23);
        float sums[NG];
#pragma unroll
        for (int k = 0; k < NG; ++k) sums[k] = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // pair k of a word: elements 2k and 2k + 1, at bits 4k; odd k meets c * 2^-20
                const float f = k & 1 ? mul * 0.0625f : mul;
                const uint32_t p = pack_f16(x[i][2 * k] * f, x[i][2 * k + 1] * f);
                qf[2 * i + (k >> 1)][k & 1] = p;
                sums[i / (NW / NG)] += (Fp16::lo(p) + Fp16::hi(p)) * (k & 1 ? 16.f : 1.f);
            }
        }
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], 1);
            sums[k] += __shfl_xor_sync(0xffffffffu, sums[k], 2);
            sums[k] *= 0x1p-24f;
            qsum[k][0] = __shfl_sync(0xffffffffu, sums[k], 8 * j);
            qsum[k][1] = __shfl_sync(0xffffffffu, sums[k], 8 * j + 4);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) qoff[c] = NG == 1 ? -8.f * qsum[0][c & 1] : 0.f;
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
#pragma unroll
            for (int c = 0; c < 4; ++c) e[k][c] = 0.f;
        }
        vs = 0x1p100f;
        vlimit = -1.f;   // below any |s'|: the first page sets E
    }

    static __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[NW])
    {
        if constexpr (NW == 4) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            w[0] = u.x, w[1] = u.y;
        }
    }

    static __device__ __forceinline__ void load_scales(const uint8_t* p, uint32_t (&w)[NG])
    {
        if constexpr (NG == 4) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else if constexpr (NG == 2) {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            w[0] = u.x, w[1] = u.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        }
    }

    // NP pages in shared memory; `valid` (1 .. 16) of a single page's tokens
    // count, all of a pair's.  Two at a time share the checks and keep two chains of products in flight.
    template <int NP>
    __device__ __forceinline__ void pages(const uint8_t* const (&st)[NP], int valid, float scale, int lane)
    {
        const int g = lane >> 2;
        float s[NP][4];
        uint32_t mv[NP][2][NG];
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            uint32_t ka[NW], kb[NW], mk[2][NG];
            load_words(st[p] + lane * NW * 4, ka);
            load_words(st[p] + (32 + lane) * NW * 4, kb);
            const uint8_t* sc = st[p] + 2 * B::kCodes + g * NG * 4;
            load_scales(sc, mk[0]);
            load_scales(sc + 8 * NG * 4, mk[1]);
            load_scales(sc + B::kScales, mv[p][0]);
            load_scales(sc + B::kScales + 8 * NG * 4, mv[p][1]);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                float acc[4];
                if constexpr (NG > 1) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[c] = -8.f * qsum[k][c & 1];
                }
#pragma unroll
                for (int i = k * (NW / NG); i < (k + 1) * (NW / NG); ++i) {
                    const uint32_t a8 = ka[i] >> 8, b8 = kb[i] >> 8;
                    if (NG == 1 && i == 0)
                        mma_f16_16816(acc, ka[i] & 0x000f000fu, kb[i] & 0x000f000fu, ka[i] & 0x00f000f0u, kb[i] & 0x00f000f0u,
                                      qf[2 * i][0], qf[2 * i][1], qoff);
                    else
                        mma_f16_16816(acc, ka[i] & 0x000f000fu, kb[i] & 0x000f000fu, ka[i] & 0x00f000f0u, kb[i] & 0x00f000f0u,
                                      qf[2 * i][0], qf[2 * i][1]);
                    mma_f16_16816(acc, a8 & 0x000f000fu, b8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x00f000f0u,
                                  qf[2 * i + 1][0], qf[2 * i + 1][1]);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float ss = T::lo(mk[t][k]), sz = T::hi(mk[t][k]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float& x = s[p][2 * t + c];
                        x = fmaf(ss, acc[2 * t + c], k == 0 ? sz * qsum[k][c] : fmaf(sz, qsum[k][c], x));
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) s[p][c] *= scale;   // and by qback where it meets m
            if (NP == 1 && valid < kPageSize) {   // slots past the end may hold anything
                if (g >= valid) {
                    s[p][0] = s[p][1] = -INFINITY;
#pragma unroll
                    for (int k = 0; k < NG; ++k) mv[p][0][k] = 0u;
                }
                if (g + 8 >= valid) {
                    s[p][2] = s[p][3] = -INFINITY;
#pragma unroll
                    for (int k = 0; k < NG; ++k) mv[p][1][k] = 0u;
                }
            }
        }
        // The references m and E move only when a score passes m by more than
        // 8 (log2 units) or a scale its limit: weights stay below 2^8, weights times scales
        // below 2^15, and most pages skip the reductions and the rescale.
        float vmax = 0.f, pm0 = -INFINITY, pm1 = -INFINITY;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            pm0 = fmaxf(pm0, fmaxf(s[p][0], s[p][2]));
            pm1 = fmaxf(pm1, fmaxf(s[p][1], s[p][3]));
#pragma unroll
            for (int k = 0; k < NG; ++k) vmax = fmaxf(vmax, fmaxf(fabsf(T::lo(mv[p][0][k])), fabsf(T::lo(mv[p][1][k]))));
        }
        pm0 *= qback[0];
        pm1 *= qback[1];
        if (__any_sync(0xffffffffu, pm0 > m[0] + 8.f || pm1 > m[1] + 8.f || vmax > vlimit)) move_references(pm0, pm1, vmax);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const float p0 = ex2(fmaf(s[p][0], qback[0], -m[0])), p1 = ex2(fmaf(s[p][1], qback[1], -m[1]));
            const float p2 = ex2(fmaf(s[p][2], qback[0], -m[0])), p3 = ex2(fmaf(s[p][3], qback[1], -m[1]));
            l[0] += p0 + p2;
            l[1] += p1 + p3;
            uint32_t va[NW], vb[NW];
            load_words(st[p] + B::kCodes + lane * NW * 4, va);
            load_words(st[p] + B::kCodes + (32 + lane) * NW * 4, vb);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const float s0 = T::lo(mv[p][0][k]) * vs, s1 = T::lo(mv[p][1][k]) * vs;
                const float z0 = T::hi(mv[p][0][k]), z1 = T::hi(mv[p][1][k]);
                z[k][0] = fmaf(p0, z0, fmaf(p2, z1, z[k][0]));
                z[k][1] = fmaf(p1, z0, fmaf(p3, z1, z[k][1]));
                // (p s')^T as the column operand: the packed pairs are 8x8 tiles
                // [token][n] in the fragment layout, their transposes are the operand.
                const uint32_t b0 = movmatrix_trans(pack_f16(p0 * s0, p1 * s0));
                const uint32_t b1 = movmatrix_trans(pack_f16(p2 * s1, p3 * s1));
                mma_f16_16816(e[k], 0xc800c800u, 0xc800c800u, 0xc800c800u, 0xc800c800u, b0, b1);   // -8 everywhere
#pragma unroll
                for (int i = k * (NW / NG); i < (k + 1) * (NW / NG); ++i) {
                    const uint32_t a8 = va[i] >> 8, b8 = vb[i] >> 8;
                    mma_f16_16816(o[2 * i], va[i] & 0x000f000fu, va[i] & 0x00f000f0u, vb[i] & 0x000f000fu, vb[i] & 0x00f000f0u, b0, b1);
                    mma_f16_16816(o[2 * i + 1], a8 & 0x000f000fu, a8 & 0x00f000f0u, b8 & 0x000f000fu, b8 & 0x00f000f0u, b0, b1);
                }
            }
        }
    }

    // m and E follow the lanes' largest scores and scale.
    __device__ __forceinline__ void move_references(float pm0, float pm1, float vmax)
    {
#pragma unroll
        for (int mask = 4; mask < 32; mask <<= 1) {
            pm0 = fmaxf(pm0, __shfl_xor_sync(0xffffffffu, pm0, mask));
            pm1 = fmaxf(pm1, __shfl_xor_sync(0xffffffffu, pm1, mask));
            vmax = fmaxf(vmax, __shfl_xor_sync(0xffffffffu, vmax, mask));
        }
        const float n0 = fmaxf(m[0], pm0), n1 = fmaxf(m[1], pm1);
        const float al0 = n0 == m[0] ? 1.f : ex2(m[0] - n0), al1 = n1 == m[1] ? 1.f : ex2(m[1] - n1);
        m[0] = n0;
        m[1] = n1;
        float r = 1.f;
        if (vmax > vlimit) {   // the same in all lanes
            const int ex = max(-100, (int)(__float_as_uint(vmax) >> 23) - 127);
            const float next = __uint_as_float((uint32_t)(127 + 6 - ex) << 23);   // takes vmax into [2^6, 2^7)
            r = next / vs;
            vs = next;
            vlimit = 128.f / next;
        }
        l[0] *= al0;
        l[1] *= al1;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            z[k][0] *= al0;
            z[k][1] *= al1;
            e[k][0] *= al0 * r;
            e[k][1] *= al1 * r;
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            o[mt][0] *= al0 * r;
            o[mt][1] *= al1 * r;
            o[mt][2] *= al0 * r;
            o[mt][3] *= al1 * r;
        }
    }

    // The sums over all lanes' tokens; o is then the unnormalised output.
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
        const float back = 1.f / vs;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int k = mt / (MT / NG);
                o[mt][c] = (o[mt][c] * (c < 2 ? 0x1p24f : 0x1p20f) + e[k][c & 1]) * back + z[k][c & 1];
            }
    }

    __device__ __forceinline__ void write_out(const AttnArgs& a, int b, int h, int lane) const
    {
        const int g = lane >> 2;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int n = 2 * (lane & 3) + c;
            if (n >= a.G) continue;
            const float inv = l[c] == 0.f ? 0.f : 1.f / l[c];
            uint16_t* out = a.out + b * a.out_stride + (int64_t)(h * a.G + n) * D + g;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const uint32_t w = T::pack(o[mt][c] * inv, o[mt][c + 2] * inv);
                out[16 * mt] = (uint16_t)w;
                out[16 * mt + 8] = (uint16_t)(w >> 16);
            }
            if (a.lse && g == 0) a.lse[(int64_t)b * a.Hq + h * a.G + n] = (m[c] + log2f(l[c])) * kLn2;
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

// One query row of a part: o elements lane * E .. of this lane, m and l.
template <int D>
struct RowSum {
    static constexpr int E = D / 32;
    float o[E], m, l;
    __device__ __forceinline__ RowSum() : m(-INFINITY), l(0.f)
    {
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = 0.f;
    }
    __device__ __forceinline__ void add(const float (&x)[E], float mx, float lx)
    {
        const float top = fmaxf(m, mx);
        const float a = m == top ? 1.f : ex2(m - top), b = mx == top ? 1.f : ex2(mx - top);
        m = top;
        l = l * a + lx * b;
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = o[i] * a + x[i] * b;
    }
    template <class T>
    __device__ __forceinline__ void write_out(const AttnArgs& a, int b, int h, int n, int lane) const
    {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        uint16_t* out = a.out + b * a.out_stride + (int64_t)(h * a.G + n) * D + lane * E;
#pragma unroll
        for (int i = 0; i < E; i += 2) *reinterpret_cast<uint32_t*>(out + i) = T::pack(o[i] * inv, o[i + 1] * inv);
        if (a.lse && lane == 0) a.lse[(int64_t)b * a.Hq + h * a.G + n] = (m + log2f(l)) * kLn2;
    }
};

template <int D, int NG, class T>
__global__ void __launch_bounds__(AttnShape<D, NG>::kWarps * 32, AttnShape<D, NG>::kCtas) attention_kernel(AttnArgs a)
{
    using S = AttnShape<D, NG>;
    using B = Kv4Block<D, NG>;
    using M = AttnSmem<D, NG>;
    constexpr int W = S::kWarps, R = S::kStages, E = D / 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t warp_pages[W];
    __shared__ int arrived[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint8_t* ring = smem + warp * S::kRing;
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + M::kBars) + warp * R;
    PartInfo* infos = reinterpret_cast<PartInfo*>(smem + M::kInfo);
    float* heads = reinterpret_cast<float*>(smem + M::kHeads);
    uint32_t* pages = reinterpret_cast<uint32_t*>(smem + M::pages(a.G));   // pages of the rows before each row
    uint32_t* costs = reinterpret_cast<uint32_t*>(smem + M::costs(a.G, a.batch));   // the same with kRowCost for each that is not empty
    uint8_t* last = smem + M::last(a.G, a.batch);                          // tokens on each row's last page
    if (lane < R) mbar_init(smem_addr(bars + lane), 1);
    fence_mbar_init();
    if (tid < 2 * W) infos[tid].b = -1;
    griddep_wait();
    griddep_launch_dependents();

    // Pages of the rows before each row.
    if (tid == 0) pages[0] = costs[0] = 0;
    uint64_t before = 0;      // pages in the low, rows that are not empty in the high 24 bits
    for (int r0 = 0; r0 < a.batch; r0 += W * 32) {
        const int r = r0 + tid;
        uint64_t sum = 0;
        if (r < a.batch) {
            const int seq = a.seq_ids ? a.seq_ids[r] : r;
            int len = seq >= 0 && seq < a.max_seqs ? a.lens[seq] : -1;
            if (len < 0 || len > a.max_pages * kPageSize) {
                if (blockIdx.x == 0) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
                len = 0;
            }
            const uint32_t n = (uint32_t)(len + kPageSize - 1) / kPageSize;
            last[r] = (uint8_t)(len - ((int)n - 1) * kPageSize);
            sum = n | (uint64_t)(n != 0) << 40;
        }
#pragma unroll
        for (int k = 1; k < 32; k <<= 1) {
            const uint64_t up = __shfl_up_sync(0xffffffffu, sum, k);
            if (lane >= k) sum += up;
        }
        if (lane == 31) warp_pages[warp] = sum;
        __syncthreads();
        uint64_t mine = before;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < warp) mine += warp_pages[w];
            before += warp_pages[w];
        }
        mine += sum;
        if (r < a.batch) {
            pages[r + 1] = (uint32_t)mine;
            costs[r + 1] = (uint32_t)mine + (uint32_t)(mine >> 40) * kRowCost;
        }
        __syncthreads();
    }
    const uint64_t all_pages = before & 0xffffffffffull;
    if (all_pages * a.H > 0x7fffffffull) {   // the same in all threads
        if (blockIdx.x == 0 && tid == 0) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
        return;
    }

    // Shares: equal parts of the list of tiles in which every (row, KV head)
    // is preceded by kRowCost empty places; the first `extra` warps take one place more.
    const uint32_t H = a.H, places = costs[a.batch] * H;
    const uint32_t warps = min(gridDim.x * W, (places + kMinShare - 1) / kMinShare);
    const uint32_t base = warps ? places / warps : 0, extra = warps ? places % warps : 0;
    auto cta_of = [&](int b, int h, uint32_t p) {   // the CTA whose share holds page p of a (row, KV head)
        const uint32_t n = pages[b + 1] - pages[b];
        const uint32_t at = costs[b] * H + h * (n + kRowCost) + kRowCost + p, long_ones = extra * (base + 1);
        return (int)((at < long_ones ? at / (base + 1) : extra + (at - long_ones) / base) / W);
    };
    auto row_of = [&](const uint32_t* sums, uint32_t x) {   // the last row with sums[row] <= x (so not empty, where x < sums[batch])
        int r0 = 0, r1 = a.batch;
        while (r1 - r0 > 1) {
            const int mid = (r0 + r1) >> 1;
            if (sums[mid] <= x) r0 = mid;
            else r1 = mid;
        }
        return r0;
    };
    uint32_t lo = 0;
    {   // lane 0: tiles before this warp's share, lane 1: up to its end
        const uint32_t w = min(blockIdx.x * W + warp + (lane & 1), warps), at = w * base + min(w, extra);
        if (w < warps) {
            const int r = row_of(costs, at / H);
            const uint32_t n = pages[r + 1] - pages[r], in_row = at - costs[r] * H, h = in_row / (n + kRowCost);
            const uint32_t off = in_row - h * (n + kRowCost);
            lo = pages[r] * H + h * n + (off > kRowCost ? off - kRowCost : 0);
        } else {
            lo = pages[a.batch] * H;
        }
    }
    const int count = (int)(__shfl_sync(0xffffffffu, lo, 1) - __shfl_sync(0xffffffffu, lo, 0));
    lo = __shfl_sync(0xffffffffu, lo, 0);
    const uint64_t policy = l2_policy_evict_first();

    auto tile_of = [&](int i) {   // tile i of this warp's share
        Tile t{nullptr, 0};
        if (i >= count) return t;
        const uint32_t at = lo + i;
        const int r0 = row_of(pages, at / H);
        const uint32_t first = pages[r0], n = pages[r0 + 1] - first, in_row = at - first * H;
        const int h = (int)(in_row / n), p = (int)(in_row - h * n);
        const int seq = a.seq_ids ? a.seq_ids[r0] : r0;
        const int32_t page = a.block_table[(int64_t)seq * a.max_pages + p];
        int valid = p == (int)n - 1 ? last[r0] : kPageSize;
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
    // The ring's stages hold two tiles each and are used in turn: tiles 2k and
    // 2k + 1 of the share lie in stage k % R.  Their copies are started by the lanes that hold the tiles.
    const uint32_t ring_at = smem_addr(ring), bars_at = smem_addr(bars);
    auto issue = [&](const uint8_t* from, int i, int stage) {
        if (!from) return;
        const uint32_t bar = bars_at + 8 * stage;
        if (!(lane & 1)) mbar_arrive_expect_tx(bar, i + 1 < count ? 2 * B::kBytes : B::kBytes);
        bulk_load(ring_at + (2 * stage + (lane & 1)) * B::kBytes, from, B::kBytes, bar, policy);
    };

    __syncwarp();
    Tile next = tile_of(lane);
    uint32_t cur = next.bits;         // of the 32 tiles in work; next: the 32 after them
    const uint8_t* from = next.src;   // the tile that this lane starts next
    if (lane < 2 * R) issue(from, lane, lane >> 1);
    State<D, NG, T> st;
    bool ok = true, begins = true;
    int stage = 0;
    uint32_t parity = 0;              // of the stages' phase: flips where the stages begin again
    auto start = [&](int src, bool first) {
        begins = first;
        const uint32_t t = __shfl_sync(0xffffffffu, cur, src);
        st.start(a, Tile::row(t), Tile::head(t), lane);
    };
    auto end = [&](int i, int src, bool ends) {
        const uint32_t t = __shfl_sync(0xffffffffu, cur, src);
        const int b = Tile::row(t), h = Tile::head(t);
        st.finish();
        if (begins && ends) {
            st.write_out(a, b, h, lane);
        } else {
            // A part that is not the share's last one began before it.
            const int k = i == count - 1 ? 1 : 0;
            __syncwarp();             // the ring's last tiles have been read
            st.write_part(k ? reinterpret_cast<float*>(ring) : heads + warp * part_floats(a.G, D), a.G, lane);
            if (lane == 0) infos[2 * warp + k] = {b, h, begins, ends};
        }
    };
    for (int i0 = 0; i0 < count; i0 += 32) {
        if (i0) cur = next.bits;
        const int here = min(32, count - i0);
        // Of the 32 tiles in cur: first and last pages; where a state starts and
        // ends; even tiles that make a pair of full pages of one row with the next one.
        const uint32_t firsts = __ballot_sync(0xffffffffu, cur & Tile::kFirst);
        const uint32_t lasts = __ballot_sync(0xffffffffu, cur & Tile::kLast);
        const uint32_t fulls = __ballot_sync(0xffffffffu, (cur & 31) == kPageSize);
        uint32_t opens = firsts | (i0 == 0 ? 1u : 0u);
        uint32_t closes = lasts | (i0 + 32 >= count ? 1u << (here - 1) : 0u);
        uint32_t pairs = fulls & (fulls >> 1) & ~lasts;
        next = tile_of(i0 + 32 + lane);
        for (int src = 0; src < here; src += 2, opens >>= 2, closes >>= 2, pairs >>= 2) {
            if (ok) {
                const uint32_t bar = bars_at + 8 * stage;
                bool w = mbar_try_wait(bar, parity);
                if (!w) w = wait_long(bar, parity);
                ok = __all_sync(0xffffffffu, w);
                if (!ok) {   // the rest of the share is left out; copies in flight land first
                    if (lane == 0) kv4_error(a.err, KVC_DEVERR_WAIT_TIMEOUT);
                    const int done = (i0 + src) / 2, all = (count + 1) / 2;
                    for (int k = done; k < min(done + R, all); ++k) mbar_wait_bounded(bars_at + 8 * (k % R), (k / R) & 1, kWaitLimitNs);
                }
            }
            const uint8_t* tile = ring + 2 * stage * B::kBytes;
            if (pairs & 1u) {
                if (opens & 1u) start(src, (firsts >> src) & 1u);
                const uint8_t* const tiles[2] = {tile, tile + B::kBytes};
                if (ok) st.pages(tiles, kPageSize, a.scale, lane);
                if (closes & 2u) end(i0 + src + 1, src + 1, (lasts >> (src + 1)) & 1u);
            } else {
#pragma unroll 1
                for (int t = 0; t < 2 && src + t < here; ++t) {
                    if ((opens >> t) & 1u) start(src + t, (firsts >> (src + t)) & 1u);
                    const uint8_t* const tiles[1] = {tile + t * B::kBytes};
                    const int valid = (int)(__shfl_sync(0xffffffffu, cur, src + t) & 31);
                    if (ok && valid) st.pages(tiles, valid, a.scale, lane);
                    if ((closes >> t) & 1u) end(i0 + src + t, src + t, (lasts >> (src + t)) & 1u);
                }
            }
            __syncwarp();
            const int to = (src + 2 * R) & 31;
            if (to == 0) from = next.src;
            if (ok && (lane >> 1) == (to >> 1)) issue(from, i0 + src + 2 * R + (lane & 1), stage);
            if (++stage == R) {
                stage = 0;
                parity ^= 1u;
            }
        }
    }

    // Rows without tokens.
    for (int r = blockIdx.x; r < a.batch; r += gridDim.x)
        if (pages[r] == pages[r + 1]) {
            for (int i = tid; i < a.Hq * (D / 8); i += W * 32)
                *reinterpret_cast<uint4*>(a.out + r * a.out_stride + i * 8) = make_uint4(0u, 0u, 0u, 0u);
            if (a.lse)
                for (int i = tid; i < a.Hq; i += W * 32) a.lse[(int64_t)r * a.Hq + i] = -INFINITY;
        }
    __syncthreads();

    // Merge this CTA's parts: one (group of adjacent parts, query row) per warp and turn.
    const int PF = part_floats(a.G, D);
    auto part_of = [&](int e) {
        return e & 1 ? reinterpret_cast<const float*>(smem + (e >> 1) * S::kRing) : heads + (e >> 1) * PF;
    };
    int turn = 0, open[2] = {-1, -1};   // entries of the groups that go on before and after this CTA
    for (int e = 0; e < 2 * W;) {
        if (infos[e].b < 0) {
            ++e;
            continue;
        }
        int f = e + 1, ends = infos[e].ends;
        for (; f < 2 * W && !ends; ++f)
            if (infos[f].b >= 0) ends = infos[f].ends;
        const PartInfo& in = infos[e];
        const int slot = in.begins ? 1 : 0;
        const bool whole = in.begins && ends;
        if (!whole) open[slot] = e;
        for (int n = 0; n < a.G; ++n, ++turn) {
            if (turn % W != warp) continue;
            RowSum<D> sum;
            for (int k = e; k < f; ++k) {
                if (infos[k].b < 0) continue;
                const float* p = part_of(k);
                float x[E];
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = p[n * D + lane * E + i];
                sum.add(x, p[a.G * D + n], p[a.G * (D + 1) + n]);
            }
            if (whole) {
                sum.template write_out<T>(a, in.b, in.h, n, lane);
            } else {
                float* to = a.parts + ((int64_t)blockIdx.x * 2 + slot) * PF;
#pragma unroll
                for (int i = 0; i < E; ++i) to[n * D + lane * E + i] = sum.o[i];
                if (lane == 0) {
                    to[a.G * D + n] = sum.m;
                    to[a.G * (D + 1) + n] = sum.l;
                }
            }
        }
        e = f;
    }
    if (open[0] < 0 && open[1] < 0) return;

    // What crosses CTAs: the last one to arrive merges it.
    auto ctas_of = [&](const PartInfo& in, int* c0, int* c1) {
        *c0 = cta_of(in.b, in.h, 0);
        *c1 = cta_of(in.b, in.h, pages[in.b + 1] - pages[in.b] - 1);
    };
    __syncthreads();
    if (tid < 2) {
        arrived[tid] = 0;
        if (open[tid] >= 0) {
            int c0, c1;
            ctas_of(infos[open[tid]], &c0, &c1);
            __threadfence();
            if (atomicAdd(a.counters + c0, 1) == c1 - c0) {
                a.counters[c0] = 0;
                arrived[tid] = 1;
            }
            __threadfence();
        }
    }
    __syncthreads();
    for (int k = 0; k < 2; ++k) {
        if (!arrived[k]) continue;
        const PartInfo& in = infos[open[k]];
        int c0, c1;
        ctas_of(in, &c0, &c1);
        for (int n = warp; n < a.G; n += W) {
            RowSum<D> sum;
            for (int c = c0; c <= c1; ++c) {
                const float* p = a.parts + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * PF;
                float x[E];
#pragma unroll
                for (int i = 0; i < E; ++i) x[i] = __ldcg(p + n * D + lane * E + i);
                sum.add(x, __ldcg(p + a.G * D + n), __ldcg(p + a.G * (D + 1) + n));
            }
            sum.template write_out<T>(a, in.b, in.h, n, lane);
        }
    }
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

constexpr int kSmemPerSm = 228 * 1024, kSmemPerCta = 1024 + 128;   // what an SM has, what a CTA takes beside its dynamic part

template <int D, int NG>
struct AttnPlan {
    using S = AttnShape<D, NG>;
    static int ctas_per_sm(int G, int batch)
    {
        const int fit = kSmemPerSm / (AttnSmem<D, NG>::bytes(G, batch) + kSmemPerCta);
        return fit < S::kCtas ? fit : S::kCtas;
    }
};

struct WorkspaceOf {
    int sms, G;
    template <int D, int NG, class T>
    int64_t operator()() const
    {
        const int64_t ctas = (int64_t)sms * AttnShape<D, NG>::kCtas;
        return 256 * ((ctas * 4 + 255) / 256) + ctas * 2 * part_floats(G, D) * 4;
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
        static OncePerDevice once;
        const int smem = AttnSmem<D, NG>::bytes(a.G, a.batch);
        constexpr int most = AttnSmem<D, NG>::bytes(kMaxGroup, kKv4MaxBatch);
        static_assert(part_floats(kMaxGroup, D) * 4 <= S::kRing, "a part lies in its warp's ring");
        static_assert(most <= 227 * 1024, "shared memory of a CTA");
        cudaError_t e = once.set_attribute(attention_kernel<D, NG, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e != cudaSuccess) return e;
        const int grid = sms * AttnPlan<D, NG>::ctas_per_sm(a.G, a.batch);
        return kv4_launch(attention_kernel<D, NG, T>, dim3((unsigned)grid), S::kWarps * 32, (size_t)smem, st, a);
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
    return kv4_dispatch(*pool, WorkspaceOf{sms, num_q_heads / pool->num_kv_heads});
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
    if (!(softmax_scale <= 0.f) && !std::isfinite(softmax_scale))
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: softmax_scale must be finite");
    if (!kv4_aligned(workspace, 256) || workspace_bytes < 256)
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: workspace must be 256-byte aligned and of kv4_workspace_bytes()");
    const int sms = device_sms();
    if (!sms) return kv4_fail(KVC_ERR_CUDA, "kv4_decode_attention: cannot query the current device");
    const int G = num_q_heads / pool->num_kv_heads;
    if (workspace_bytes < kv4_dispatch(*pool, WorkspaceOf{sms, G}))
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: the workspace is smaller than kv4_workspace_bytes()");
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)pool->head_dim);
    AttnArgs a{};
    a.pool = static_cast<const uint8_t*>(pool->data);
    a.num_pages = pool->num_pages;
    a.H = pool->num_kv_heads;
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
    a.scale = scale * 1.4426950408889634f * 0x1p24f;
    a.err = device_error;
    const int64_t most = (int64_t)sms * kCtasPerSm * 4;
    a.counters = static_cast<int32_t*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + 256 * ((most + 255) / 256));
    return kv4_launch_result(kv4_dispatch(*pool, LaunchAttention{a, sms, static_cast<cudaStream_t>(stream)}));
}
