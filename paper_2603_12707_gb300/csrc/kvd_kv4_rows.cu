// kv4_write and kv4_read: K and V rows of tokens into and out of the 4-bit
// pool's blocks (layout and quantisation: kvdecode4.h).  Both are copies whose
// one side is 16-bit rows and whose other side is blocks.
//
// V's codes lie in words of two neighbouring tokens, so a warp takes tokens
// whose slots 2m and 2m + 1 follow one another as a pair (a run of tokens gives
// pairs wherever it starts) and others alone; it goes over some KV heads of
// them.  A lane holds 8 consecutive elements of one token's row, which are one word of K's
// codes; V's words hold elements 8 apart, four lanes' codes each, and are made by a transposition across lanes.
//
// Measured on 57344 tokens of 32 heads of 128, groups of 64, bf16 (1.20 GB each
// way, 177 us at the speed of a copy): kv4_write 247 us, 4.9 TB/s, bound by the
// instructions (254 for a pair's head; the schedulers issue 77 % of cycles, the ALU pipe is 66 % busy);
// kv4_read 197 us, 6.1 TB/s, bound by memory.  32 warps an SM (64
// registers) do better than 24 in both.  A call for 64 tokens takes 2.6 and 2.1 us of the device.
#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kRowWarps = 8;

struct RowsArgs {
    uint8_t* pool;
    int64_t num_slots;     // num_pages * 16
    int32_t H, n;
    int32_t warp_heads;    // KV heads that a warp goes over
    const int64_t* slots;
    uint16_t* k;           // [n][H][D], row strides k_stride and v_stride
    uint16_t* v;
    int64_t k_stride, v_stride;
    int32_t* err;
};

// A turn's tokens: t alone, or t and t + 1 in slots 2m and 2m + 1.
struct Turn {
    int64_t slot;
    int tokens;     // 0: the token before takes it along
    bool known;     // the slot is one of the pool's
};

__device__ __forceinline__ Turn turn_of(const RowsArgs& a, int64_t t, bool report)
{
    const int64_t s = a.slots[t], before = t > 0 ? a.slots[t - 1] : -2, after = t + 1 < a.n ? a.slots[t + 1] : -2;
    const bool known = s >= 0 && s < a.num_slots, odd = s & 1;
    if (!known && s != -1 && report) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
    return {s, known && odd && before == s - 1 ? 0 : known && !odd && after == s + 1 ? 2 : 1, known};
}

// 4 x 4 bytes across the lanes of a quad: lane n gets byte n of lanes 0 .. 3.
__device__ __forceinline__ uint32_t quad_transpose(uint32_t w, int lane)
{
    w = __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 1), lane & 1 ? 0x3715 : 0x6240);
    return __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 2), lane & 2 ? 0x3276 : 0x5410);
}

// The low nibbles of four bytes, as 16 bits (nibble n of lane n's byte).
__device__ __forceinline__ uint32_t low_nibbles(uint32_t w)
{
    w &= 0x0f0f0f0fu;
    w = (w | w >> 4) & 0x00ff00ffu;
    return (w | w >> 8) & 0xffffu;
}

template <class T>
struct Packed;
template <>
struct Packed<Bf16> {
    using V = __nv_bfloat162;
    static constexpr uint32_t kMagic = 0x43004300u;    // 128 + code in the low bits
    static constexpr float kOffset = -136.f;           // ... to code - 8
    static constexpr bool kTiny = true;                // holds numbers whose reciprocal fp32 does not
    static __device__ __forceinline__ V dup(float x) { return __float2bfloat162_rn(x); }
};
template <>
struct Packed<Fp16> {
    using V = __half2;
    static constexpr uint32_t kMagic = 0x64006400u;    // 1024 + code
    static constexpr float kOffset = -1032.f;
    static constexpr bool kTiny = false;
    static __device__ __forceinline__ V dup(float x) { return __float2half2_rn(x); }
};
template <class V>
__device__ __forceinline__ V as_pair(uint32_t w)
{
    return *reinterpret_cast<const V*>(&w);
}
template <class V>
__device__ __forceinline__ uint32_t as_word(V v)
{
    return *reinterpret_cast<const uint32_t*>(&v);
}

// s (c - 8) + z of two codes (bits 0-3 and 16-19 of `codes`): one rounding, in the cache's type.
template <class T>
__device__ __forceinline__ uint32_t dequantise(uint32_t codes, typename Packed<T>::V s, typename Packed<T>::V z)
{
    using V = typename Packed<T>::V;
    const V c = __hadd2(as_pair<V>((codes & 0x000f000fu) | Packed<T>::kMagic), Packed<T>::dup(Packed<T>::kOffset));
    return as_word(__hfma2(c, s, z));
}

// (min, -max) of this lane's 8 elements, in the cache's type: one minimum serves both.
template <class T>
__device__ __forceinline__ uint32_t range_of(const uint4& row)
{
    using V = typename Packed<T>::V;
    const uint32_t w[4] = {row.x, row.y, row.z, row.w};
    V lo = as_pair<V>(w[0]), hi = lo;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        lo = __hmin2_nan(lo, as_pair<V>(w[i]));
        hi = __hmax2_nan(hi, as_pair<V>(w[i]));
    }
    const uint32_t l = as_word(lo), h = as_word(__hneg2(hi));
    return as_word(__hmin2_nan(as_pair<V>(__byte_perm(l, h, 0x5410)), as_pair<V>(__byte_perm(l, h, 0x7632))));
}

constexpr uint32_t kBroken = 0x7fff7fffu;     // the scale word of a group with an infinity or a NaN: NaN in either type

// bf16's tiny steps are scaled up, exactly, so that 1 / s is finite (elements are tiny then, too; a step of
// 0 may have large ones, which would overflow).
template <class T>
__device__ __forceinline__ float scale_up(float s)
{
    return Packed<T>::kTiny && s < 0x1p-100f && s > 0.f ? 0x1p64f : 1.f;
}

// The scale word (s, z) of a group's (min, -max), and 1 / s (scaled down by scale_up; 0 for a
// step of 0, which makes every quotient 0).
//
// Where z + 7 s or z - 8 s would round to an infinity, s is the next smaller number and z is rounded toward
// zero.  Then 15 s is at least 7.5 units of s below max - min, so the top is below max where z > 0; where z < 0 the top would
// need 7 s past the type's range, which 15 s has.  The bottom is at least min where z < 0; where z > 0 it is
// less than a unit of z below, and s is above an eighth of the range there, z below a fifteenth.
template <class T>
__device__ __forceinline__ uint32_t scale_of(uint32_t range, float* r)
{
    const float least = T::lo(range), most = -T::hi(range);
    const float half = most * 0.5f - least * 0.5f;
    // half / 7.5, corrected once like the quotients below.
    const float h0 = half * (1.f / 7.5f);
    uint32_t step = T::pack(fmaf(fmaf(-7.5f, h0, half), 1.f / 7.5f, h0), 0.f);
    float s = T::lo(step);
    uint32_t middle = T::pack(fmaf(8.f, s, least), 0.f);
    if (fmaxf(most, -least) > T::kNear && (fmaf(7.f, s, T::lo(middle)) >= T::kOver || fmaf(-8.f, s, T::lo(middle)) <= -T::kOver)) {
        s = T::lo(--step);
        middle = T::toward_zero(fmaf(8.f, s, least));
    }
    *r = s > 0.f ? 1.f / (s * scale_up<T>(s)) : 0.f;
    return half < INFINITY ? __byte_perm(step, middle, 0x5410) : kBroken;
}

// The codes of this lane's 8 elements, as K's words hold them (element e in
// bits 16 (e % 2) + 4 (e / 2) and up).
//
// The quotient.  With r = 1 / s, k = rint(d r) is the nearest code or, close to a tie,
// its neighbour; e = d - k s is exact and k + e r is d / s but for one rounding,
// on a tie exactly the tie.  It is at most some 50 (z is off by half a unit of its
// type, and s at least a thirtieth of one where it is not 0), so 16 bits hold it until
// the clamp.  (Where d overflows, at -8 s of the widest groups that bf16 holds,
// it is NaN, whose bits the clamp takes to 0 as it should.)
template <class T>
__device__ __forceinline__ uint32_t quantise(const uint4& row, uint32_t scale, float r)
{
    const uint32_t w[4] = {row.x, row.y, row.z, row.w};
    const float s = T::lo(scale), z = T::hi(scale), up = scale_up<T>(s), su = s * up;
    constexpr float kRound = 12582912.f;      // 1.5 * 2^23: adding it rounds to an integer, in the low bits
    const uint64_t up2 = f2_pack(up, up), z2 = f2_pack(-z * up, -z * up), s2 = f2_pack(-su, -su), r2 = f2_pack(r, r);
    const uint64_t round2 = f2_pack(kRound, kRound), back2 = f2_pack(-kRound, -kRound), code2 = f2_pack(kRound + 8.f, kRound + 8.f);
    uint32_t codes = 0;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
        const uint64_t x = f2_pack(T::lo(w[i]), T::hi(w[i]));
        const uint64_t d = Packed<T>::kTiny ? f2_fma(x, up2, z2) : f2_add(x, z2);
        const uint64_t k = f2_add(f2_fma(d, r2, round2), back2);
        float q0, q1;
        f2_unpack(f2_add(f2_fma(f2_fma(k, s2, d), r2, k), code2), q0, q1);
        const uint32_t c = __vimin_s16x2_relu(__byte_perm(__float_as_uint(q0), __float_as_uint(q1), 0x5410), 0x000f000fu);
        codes = codes * 16u + c;
    }
    return scale == kBroken ? 0x88888888u : codes;
}

// Byte offsets in a block.
template <int D>
__device__ __forceinline__ int v_word_offset(int tok, int g, int i)   // of the word that holds token tok
{
    return ((((tok >> 3) * 8 + g) * 4 + ((tok & 7) >> 1)) * (D / 32) + i) * 4;
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N])
{
    if constexpr (N == 4) {
        const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
    } else if constexpr (N == 2) {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(p));
        w[0] = x.x, w[1] = x.y;
    } else {
        w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    }
}

// A lane's part of one step over HS heads: rows are (token of the turn, head)
// in D / 8 lanes each, tokens 16 lanes apart.
template <int D>
struct Place {
    static constexpr int HS = 128 / D;   // heads of a step
    int second, head, m;                 // token of the turn, head of the step, 8-element part of the row
    __device__ __forceinline__ explicit Place(int lane) : second(lane >> 4), head((lane & 15) / (D / 8)), m(lane % (D / 8)) {}
};

template <int D, int NG, class T>
__global__ void __launch_bounds__(kRowWarps * 32, 4) write_kernel(RowsArgs a)
{
    using B = Kv4Block<D, NG>;
    constexpr int GL = D / NG / 8, HS = Place<D>::HS, NW = D / 32;
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    const Place<D> at(lane);
    const int h0 = blockIdx.y * a.warp_heads, h1 = min(a.H, h0 + a.warp_heads);
    const int64_t first = ((int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5)) * 2;
#pragma unroll 1
    for (int64_t t = first; t < min(first + 2, (int64_t)a.n); ++t) {
        const Turn turn = turn_of(a, t, lane == 0 && blockIdx.y == 0);
        if (!turn.known || turn.tokens == 0) continue;
        const bool pair = turn.tokens == 2;
        const int tok0 = (int)(turn.slot & (kPageSize - 1)), tok = tok0 + (pair ? at.second : 0);
        uint8_t* const page = a.pool + (turn.slot >> 4) * a.H * B::kBytes;
        const int64_t row = t + (pair ? at.second : 0);
        const bool mine = pair || at.second == 0;
        const uint16_t* const k_row = a.k + row * a.k_stride + at.m * 8;
        const uint16_t* const v_row = a.v + row * a.v_stride + at.m * 8;
        uint4 k_next = make_uint4(0u, 0u, 0u, 0u), v_next = k_next;
        if (mine && h0 + at.head < h1) {
            k_next = __ldcs(reinterpret_cast<const uint4*>(k_row + (h0 + at.head) * D));
            v_next = __ldcs(reinterpret_cast<const uint4*>(v_row + (h0 + at.head) * D));
        }
#pragma unroll 1
        for (int h = h0; h < h1; h += HS) {
            const int head = h + at.head;
            const bool on = mine && head < h1;
            const uint4 kr = k_next, vr = v_next;
            if (mine && head + HS < h1) {   // the next head's rows come while these are worked
                k_next = __ldcs(reinterpret_cast<const uint4*>(k_row + (head + HS) * D));
                v_next = __ldcs(reinterpret_cast<const uint4*>(v_row + (head + HS) * D));
            }
            uint8_t* const block = page + (int64_t)head * B::kBytes;
            // Groups lie in GL lanes, whose even ones work out K's scale and whose odd ones V's (both in every lane: 255 us for 240).
            using V = typename Packed<T>::V;
            const bool odd = lane & 1;
            const uint32_t k_range = range_of<T>(kr), v_range = range_of<T>(vr);
            V range = __hmin2_nan(as_pair<V>(odd ? v_range : k_range), as_pair<V>(__shfl_xor_sync(0xffffffffu, odd ? k_range : v_range, 1)));
#pragma unroll
            for (int k = 2; k < GL; k <<= 1) range = __hmin2_nan(range, as_pair<V>(__shfl_xor_sync(0xffffffffu, as_word(range), k)));
            float r;
            const uint32_t scale = scale_of<T>(as_word(range), &r), scale_x = __shfl_xor_sync(0xffffffffu, scale, 1);
            const float r_x = __shfl_xor_sync(0xffffffffu, r, 1);
            const uint32_t ks = odd ? scale_x : scale, vs = odd ? scale : scale_x;
            const uint32_t kw = quantise<T>(kr, ks, odd ? r_x : r);
            const uint32_t vc = quad_transpose(quantise<T>(vr, vs, odd ? r : r_x), lane);
            // Lane (i, n) of a token now holds byte n of the four lanes of word
            // i: their elements g and, in the high nibbles, g + 2.
            const int i = at.m >> 2, g = (at.m & 1) * 4 + (at.m >> 1 & 1);
            const uint32_t v = low_nibbles(vc) | low_nibbles(vc >> 4) << 16;
            const uint32_t other = __shfl_xor_sync(0xffffffffu, v, 16);
            if (on) {
                reinterpret_cast<uint32_t*>(block)[(tok * 4 + (at.m & 3)) * NW + (at.m >> 2)] = kw;
                if (at.m % GL == 0) {
                    uint32_t* scales = reinterpret_cast<uint32_t*>(block + 2 * B::kCodes) + tok * NG + at.m / GL;
                    scales[0] = ks;
                    scales[kPageSize * NG] = vs;
                }
                uint8_t* const vcodes = block + B::kCodes;
                if (pair) {   // the first token's lanes write g, the second's g + 2
                    const uint32_t word = at.second ? __byte_perm(other, v, 0x7632) : __byte_perm(v, other, 0x5410);
                    *reinterpret_cast<uint32_t*>(vcodes + v_word_offset<D>(tok0, g + 2 * at.second, i)) = word;
                } else {
                    uint8_t* const to = vcodes + v_word_offset<D>(tok, g, i) + (tok & 1) * 2;
                    *reinterpret_cast<uint16_t*>(to) = (uint16_t)v;
                    *reinterpret_cast<uint16_t*>(to + 2 * 4 * NW * 4) = (uint16_t)(v >> 16);
                }
            }
        }
    }
}

template <int D, int NG, class T>
__global__ void __launch_bounds__(kRowWarps * 32, D == 128 && NG <= 2 ? 4 : 3) read_kernel(RowsArgs a)
{
    using B = Kv4Block<D, NG>;
    using V = typename Packed<T>::V;
    constexpr int GL = D / NG / 8, HS = Place<D>::HS, NW = D / 32;
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31;
    const Place<D> at(lane);
    const int h0 = blockIdx.y * a.warp_heads, h1 = min(a.H, h0 + a.warp_heads);
    const int64_t first = ((int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5)) * 2;
#pragma unroll 1
    for (int64_t t = first; t < min(first + 2, (int64_t)a.n); ++t) {
        const Turn turn = turn_of(a, t, lane == 0 && blockIdx.y == 0);
        if (turn.tokens == 0) continue;
        const bool pair = turn.tokens == 2;
        if (!turn.known) {
            for (int h = h0; h < h1; h += HS)
                if (at.second == 0 && h + at.head < h1) {
                    reinterpret_cast<uint4*>(a.k + t * a.k_stride + (h + at.head) * D)[at.m] = make_uint4(0u, 0u, 0u, 0u);
                    reinterpret_cast<uint4*>(a.v + t * a.v_stride + (h + at.head) * D)[at.m] = make_uint4(0u, 0u, 0u, 0u);
                }
            continue;
        }
        const int tok0 = (int)(turn.slot & (kPageSize - 1)), tok = tok0 + (pair ? at.second : 0);
        const bool mine = pair || at.second == 0;
        const uint8_t* const page = a.pool + (turn.slot >> 4) * a.H * B::kBytes;
        // K: a word of a token's row per lane.  V: lane (g, j) takes elements
        // 32 i + 8 j + g of both tokens; the 8x8 tile [g][(j, token)] transposed
        // gives lane ((j, token), c) elements 32 i + 8 j + 2c and 2c + 1 of one token.
        const int g = lane >> 2, j = lane & 3;
        const bool stored = pair || (g & 1) == (tok0 & 1);
        uint16_t* const k_out = a.k + (t + at.second) * a.k_stride + at.m * 8;
        uint16_t* const v_out = a.v + (t + (pair ? g & 1 : 0)) * a.v_stride + 8 * (g >> 1) + 2 * j;
        struct Step {   // what a lane needs of one step
            uint32_t k, ks, v[HS][NW], vs[HS][2][NG];
        };
        auto load = [&](int h) {
            Step x = {};
            if (mine && h + at.head < h1) {
                const uint8_t* block = page + (int64_t)(h + at.head) * B::kBytes;
                x.k = __ldg(reinterpret_cast<const uint32_t*>(block) + (tok * 4 + (at.m & 3)) * NW + (at.m >> 2));
                x.ks = __ldg(reinterpret_cast<const uint32_t*>(block + 2 * B::kCodes) + tok * NG + at.m / GL);
            }
#pragma unroll
            for (int u = 0; u < HS; ++u) {
                if (h + u >= h1) break;
                const uint8_t* block = page + (int64_t)(h + u) * B::kBytes;
                load_words(block + B::kCodes + v_word_offset<D>(tok0, g, 0), x.v[u]);
                const uint8_t* scales = block + 2 * B::kCodes + B::kScales + (tok0 & ~1) * NG * 4;
                load_words(scales, x.vs[u][0]);
                load_words(scales + NG * 4, x.vs[u][1]);
            }
            return x;
        };
        auto store = [&](const Step& x, int h) {
            if (mine && h + at.head < h1) {
                const V s = as_pair<V>(__byte_perm(x.ks, x.ks, 0x1010)), z = as_pair<V>(__byte_perm(x.ks, x.ks, 0x3232));
                __stcs(reinterpret_cast<uint4*>(k_out + (h + at.head) * D),
                       make_uint4(dequantise<T>(x.k, s, z), dequantise<T>(x.k >> 4, s, z), dequantise<T>(x.k >> 8, s, z), dequantise<T>(x.k >> 12, s, z)));
            }
#pragma unroll
            for (int u = 0; u < HS; ++u) {
                if (h + u >= h1) break;
#pragma unroll
                for (int i = 0; i < NW; ++i) {
                    const uint32_t m0 = x.vs[u][0][i / (NW / NG)], m1 = x.vs[u][1][i / (NW / NG)];
                    const uint32_t y = movmatrix_trans(dequantise<T>(x.v[u][i] >> (4 * j), as_pair<V>(__byte_perm(m0, m1, 0x5410)),
                                                                     as_pair<V>(__byte_perm(m0, m1, 0x7632))));
                    if (stored) __stcs(reinterpret_cast<uint32_t*>(v_out + (h + u) * D + 32 * i), y);
                }
            }
        };
        // Two steps' loads are under way while two are worked.
        Step next0 = load(h0), next1 = load(h0 + HS);
#pragma unroll 1
        for (int h = h0; h < h1; h += 2 * HS) {
            const Step x0 = next0, x1 = next1;
            next0 = load(h + 2 * HS);
            next1 = load(h + 3 * HS);
            store(x0, h);
            store(x1, h + HS);
        }
    }
}

template <bool kWrite>
struct LaunchRows {
    RowsArgs& a;
    cudaStream_t st;
    template <int D, int NG, class T>
    cudaError_t operator()() const
    {
        // A warp goes over as many heads as leave every SM some 32 warps of work: a
        // warp's start is two trips to memory, slots and rows, that nothing hides (32
        // heads of 57344 tokens: 252 us at 8 heads a warp, 240 at 32; reading, 208 and 196).
        // Several pairs of tokens a warp, as one run or 16 tokens apart, are 5 to 15 % slower.
        const int64_t turns = ((int64_t)a.n + 1) / 2;
        int heads = Place<D>::HS;
        while (heads < a.H && turns * ((a.H + 2 * heads - 1) / (2 * heads)) >= 152 * 32) heads *= 2;
        a.warp_heads = heads;
        const dim3 grid((unsigned)((turns + kRowWarps - 1) / kRowWarps), (unsigned)((a.H + heads - 1) / heads));
        return kv4_launch(kWrite ? write_kernel<D, NG, T> : read_kernel<D, NG, T>, grid, kRowWarps * 32, 0, st, a);
    }
};

int rows_call(bool write, const kv4_pool* pool, int32_t n, const int64_t* slots, const void* k, int64_t k_stride,
              const void* v, int64_t v_stride, int32_t* device_error, void* stream)
{
    if (int rc = kv4_check_pool(pool, true)) return rc;
    if (n < 0) return kv4_fail(KVC_ERR_INVALID, "kv4 rows: n must be >= 0");
    if (n == 0) return KVC_OK;
    if (!slots || !k || !v) return kv4_fail(KVC_ERR_INVALID, "kv4 rows: null argument");
    if (!kv4_aligned(slots, 8) || !kv4_aligned(k, 16) || !kv4_aligned(v, 16) || k_stride % 8 || v_stride % 8)
        return kv4_fail(KVC_ERR_INVALID, "kv4 rows: rows must be 16-byte aligned, strides multiples of 8 elements");
    const int64_t least = write ? 0 : (int64_t)pool->num_kv_heads * pool->head_dim;
    if (n > 1 && (k_stride < least || v_stride < least))
        return kv4_fail(KVC_ERR_INVALID, write ? "kv4_write: strides must be >= 0" : "kv4_read: rows overlap");
    RowsArgs a{};
    a.pool = static_cast<uint8_t*>(pool->data);
    a.num_slots = pool->num_pages * kPageSize;
    a.H = pool->num_kv_heads;
    a.n = n;
    a.slots = slots;
    a.k = static_cast<uint16_t*>(const_cast<void*>(k));
    a.v = static_cast<uint16_t*>(const_cast<void*>(v));
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.err = device_error;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return kv4_launch_result(write ? kv4_dispatch(*pool, LaunchRows<true>{a, st}) : kv4_dispatch(*pool, LaunchRows<false>{a, st}));
}

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int64_t kv4_pool_bytes(const kv4_pool* pool)
{
    if (int rc = kv4_check_pool(pool, false)) return rc;
    return pool->num_pages * pool->num_kv_heads * kv4_block_bytes(*pool);
}

extern "C" KVC_API int kv4_write(const kv4_pool* pool, int32_t n, const int64_t* slots, const void* k, int64_t k_stride,
                                 const void* v, int64_t v_stride, int32_t* device_error, void* stream)
{
    return rows_call(true, pool, n, slots, k, k_stride, v, v_stride, device_error, stream);
}

extern "C" KVC_API int kv4_read(const kv4_pool* pool, int32_t n, const int64_t* slots, void* k_out, int64_t k_stride,
                                void* v_out, int64_t v_stride, int32_t* device_error, void* stream)
{
    return rows_call(false, pool, n, slots, k_out, k_stride, v_out, v_stride, device_error, stream);
}
