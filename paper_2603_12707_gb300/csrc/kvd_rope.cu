// kv_qk_rope and kv16_write: norms of queries and keys for each head, their
// rotation by positions, and the write of keys and values into a paged cache
// (kvdecode16.h), one pass over the rows.
//
// A head's row lies over D / 16 lanes, each with two chunks of 8 elements that
// hold both sides of its pairs: the rotation needs no exchange, the norm's sum
// one over those lanes.  A lane works out the angles of its 8 pairs once for
// its token and uses them for all heads that the warp goes over.  The angle is a
// whole number of 2^-64 turns (position times frequency modulo 2^64), of which
// the upper 32 bits go into the sine.
//
// Bound by memory where there are many rows: 49152 tokens of 28 + 4 heads, in and out, 121 us (6.6 TB/s), 40960 tokens of
// 32 + 2 x 32 heads into pages 311 us (6.5 TB/s).  A chunk of 5003 normed tokens of 24 heads takes 12.6 us (4.9 TB/s: a wave of warps and a
// part of one, each two trips to memory long, a third of the time instructions), 32 tokens 2.0 us (the launch and those trips).  A warp goes over a part of its token's heads, kAhead
// turns of rows under way; few tokens are shared among more warps.
#include <string>

#include "kvd_kv16.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kRopeWarps = 1;      // of a CTA, so that a token's end frees its place (5003 normed tokens of 24 heads 13.1 us with 4, 12.6 with 1)
constexpr int kAhead = 3;      // turns whose rows are under way together (2: that chunk 13.1 us; 4: 12.3, but 64 tokens into pages 3.1 instead of 2.95)

struct RopeArgs {
    const uint64_t* freqs;
    const uint8_t* axes;
    const int32_t* positions;
    int64_t axis_stride;
    int32_t num_axes, rot_chunks;     // chunks of 8 pairs
    float scale, eps;
    int32_t n, hq, hkv, parts, part_heads;
    const uint16_t *q, *k, *v;        // v: writes into the pool
    uint16_t *q_out, *k_out;          // k_out: rows, or the K pool
    uint16_t* v_out;                  // the V pool
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    const uint16_t *q_weight, *k_weight;
    const int64_t* slots;
    int64_t num_slots;
    int32_t* err;
};

enum RopeKind { kNoRotation, kHalves, kNeighbours };

template <class T>
__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8])
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = T::lo(u[i]);
        x[2 * i + 1] = T::hi(u[i]);
    }
}

template <class T>
__device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    return make_uint4(T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7]));
}

// 1 / sqrt(mean of squares + eps) of a head's elements, which makes them 2^-96 times as large where they are normed and their
// squares pass the range of 32 bits.
template <int D>
__device__ __forceinline__ float norm_of(float (&a)[8], float (&b)[8], float eps, bool normed)
{
    uint64_t u = 0ull, v = 0ull;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const uint64_t p = f2_pack(a[i], a[i + 1]), q = f2_pack(b[i], b[i + 1]);
        u = f2_fma(p, p, u);
        v = f2_fma(q, q, v);
    }
    float s, z;
    f2_unpack(f2_add(u, v), s, z);
    s += z;
#pragma unroll
    for (int m = 1; m < D / 16; m <<= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    float r = rsqrtf(fmaf(s, 1.f / D, eps));
    const bool far = normed && s > 0x1p126f;
    if (__any_sync(0xffffffffu, far)) {
        const float by = far ? 0x1p-96f : 1.f;
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] *= by;
            b[i] *= by;
            t = fmaf(a[i], a[i], fmaf(b[i], b[i], t));
        }
#pragma unroll
        for (int m = 1; m < D / 16; m <<= 1) t += __shfl_xor_sync(0xffffffffu, t, m);
        if (far) r = rsqrtf(t * (1.f / D));
    }
    return r;
}

// Sine and cosine of `turn` / 2^32 turns: the nearest quarter turn, and Taylor's series of what is left, at most pi / 4, to
// terms below 2^-25.
__device__ __forceinline__ void sine_cosine(uint32_t turn, float* sine, float* cosine)
{
    const uint32_t quarter = (turn + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(turn - (quarter << 30)) * 1.46291807926715968e-9f;   // 2 pi / 2^32
    const float y = x * x;
    const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), x);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.f);
    const float u = quarter & 1 ? c : s, v = quarter & 1 ? s : c;
    *sine = __uint_as_float(__float_as_uint(u) ^ (quarter & 2) << 30);
    *cosine = __uint_as_float(__float_as_uint(v) ^ ((quarter + 1) & 2) << 30);
}

__device__ __forceinline__ uint4 load_row(const uint16_t* p)   // (read once; not kept in L1, since the same rows may be written)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

template <int D, class T, RopeKind KIND, bool NORM, bool POOL>
__global__ void __launch_bounds__(32 * kRopeWarps) rope_kernel(RopeArgs a)
{
    constexpr int kLanes = D / 16, kHeads = 32 / kLanes;   // lanes of a head; heads at a time
    griddep_wait();
    griddep_launch_dependents();
    const int64_t w = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, sub = lane % kLanes;
    const int64_t t = a.parts == 1 ? w : w / a.parts;
    if (t >= a.n) return;
    const int first = (int)(w - t * a.parts) * a.part_heads;
    const int heads = a.hq + (POOL ? 2 : 1) * a.hkv, stop = min(first + a.part_heads, heads);

    // This lane's chunks, and the rows' addresses; the first rows are under way while the angles are worked out.
    const int rc = KIND == kNoRotation ? 0 : a.rot_chunks;
    const bool turns = KIND != kNoRotation && sub < rc;
    const int c0 = sub < rc ? sub : rc + sub, c1 = c0 + (sub < rc ? rc : kLanes - rc);
    auto source = [&](int h) {
        return h < a.hq                     ? a.q + t * a.q_stride + (int64_t)h * D
               : !POOL || h < a.hq + a.hkv ? a.k + t * a.k_stride + (int64_t)(h - a.hq) * D
                                           : a.v + t * a.v_stride + (int64_t)(h - a.hq - a.hkv) * D;
    };
    uint4 x0[kAhead], x1[kAhead];
    auto load = [&](int h0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * kHeads + lane / kLanes;
            if (h < stop) {
                const uint16_t* const src = source(h);
                x0[i] = load_row(src + c0 * 8);
                x1[i] = load_row(src + c1 * 8);
            }
        }
    };
    load(first);
    constexpr uint32_t kOnes = std::is_same_v<T, Bf16> ? 0x3f803f80u : 0x3c003c00u;   // (where only one of the two is normed)
    int64_t slot = 0;
    if (POOL) {
        slot = a.slots[t];
        if (slot < 0 || slot >= a.num_slots) {
            if (slot != -1 && lane == 0 && first == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
            slot = -1;
        }
    }
    float cs[8], sn[8];
    if (KIND != kNoRotation && turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = KIND == kHalves ? 8 * sub + i : 4 * (i < 4 ? c0 : c1) + (i & 3);
            const int axis = a.axes ? min((int)a.axes[j], a.num_axes - 1) : 0;
            const int64_t pos = a.positions[axis * a.axis_stride + t];
            sine_cosine((uint32_t)((uint64_t)pos * a.freqs[j] >> 32), &sn[i], &cs[i]);
            sn[i] *= a.scale;
            cs[i] *= a.scale;
        }
    }
    const int64_t slot_row = POOL ? ((slot / kPageSize) * a.hkv * kPageSize + slot % kPageSize) * D : 0;
#pragma unroll 1
    for (int h0 = first; h0 < stop; h0 += kAhead * kHeads) {
        if (h0 != first) load(h0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = h0 + i * kHeads + lane / kLanes;
            if (h0 + i * kHeads >= stop) break;            // (of the whole warp)
            const bool is_q = h < a.hq, is_v = POOL && h >= a.hq + a.hkv;
            const bool normed = NORM && !is_v && (is_q ? a.q_weight : a.k_weight) != nullptr;
            if (NORM || KIND != kNoRotation) {
                float x[8], y[8];
                unpack8<T>(x0[i], x);
                unpack8<T>(x1[i], y);
                if (NORM && __any_sync(0xffffffffu, normed)) {
                    const float z = norm_of<D>(x, y, a.eps, normed), f = normed ? z : 1.f;   // (values are not stored from here)
                    const uint64_t f2 = f2_pack(f, f);
                    const uint4* const weight = reinterpret_cast<const uint4*>(is_q ? a.q_weight : a.k_weight);
                    uint4 w0 = make_uint4(kOnes, kOnes, kOnes, kOnes), w1 = w0;
                    if (normed) {
                        w0 = __ldg(weight + c0);
                        w1 = __ldg(weight + c1);
                    }
                    float g[8];
                    unpack8<T>(w0, g);
#pragma unroll
                    for (int k = 0; k < 4; ++k) f2_unpack(f2_mul(f2_mul(f2_pack(x[2 * k], x[2 * k + 1]), f2), f2_pack(g[2 * k], g[2 * k + 1])), x[2 * k], x[2 * k + 1]);
                    unpack8<T>(w1, g);
#pragma unroll
                    for (int k = 0; k < 4; ++k) f2_unpack(f2_mul(f2_mul(f2_pack(y[2 * k], y[2 * k + 1]), f2), f2_pack(g[2 * k], g[2 * k + 1])), y[2 * k], y[2 * k + 1]);
                }
                if (turns) {
                    if (KIND == kHalves) {
                        if constexpr (NORM) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint64_t u = f2_pack(x[2 * k], x[2 * k + 1]), v = f2_pack(y[2 * k], y[2 * k + 1]);
                            const uint64_t c = f2_pack(cs[2 * k], cs[2 * k + 1]), z = f2_pack(sn[2 * k], sn[2 * k + 1]);
                            f2_unpack(f2_fma(u, c, f2_mul(v, f2_pack(-sn[2 * k], -sn[2 * k + 1]))), x[2 * k], x[2 * k + 1]);
                            f2_unpack(f2_fma(v, c, f2_mul(u, z)), y[2 * k], y[2 * k + 1]);
                        }
                        } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float u = x[k], v = y[k];
                            x[k] = u * cs[k] - v * sn[k];
                            y[k] = v * cs[k] + u * sn[k];
                        }
                        }
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float u = x[2 * k], v = x[2 * k + 1], u2 = y[2 * k], v2 = y[2 * k + 1];
                            x[2 * k] = u * cs[k] - v * sn[k];
                            x[2 * k + 1] = v * cs[k] + u * sn[k];
                            y[2 * k] = u2 * cs[4 + k] - v2 * sn[4 + k];
                            y[2 * k + 1] = v2 * cs[4 + k] + u2 * sn[4 + k];
                        }
                    }
                }
                if (!is_v && (turns || normed)) {
                    x0[i] = pack8<T>(x);
                    x1[i] = pack8<T>(y);
                }
            }
            if (h >= stop || (POOL && !is_q && slot < 0)) continue;
            const int kh = h - a.hq - (is_v ? a.hkv : 0);
            uint16_t* dst;
            if (is_q) dst = a.q_out + t * a.q_out_stride + (int64_t)h * D;
            else if (POOL) dst = (is_v ? a.v_out : a.k_out) + slot_row + (int64_t)kh * (kPageSize * D);
            else dst = a.k_out + t * a.k_out_stride + (int64_t)kh * D;
            reinterpret_cast<uint4*>(dst)[c0] = x0[i];
            reinterpret_cast<uint4*>(dst)[c1] = x1[i];
        }
    }
}

template <int D, class T, bool POOL>
cudaError_t launch_rope(RopeArgs& a, int kind, cudaStream_t st)
{
    constexpr int kHeads = 32 / (D / 16);
    const int heads = a.hq + (POOL ? 2 : 1) * a.hkv;
    // A warp goes over all heads of its token, whose angles it works out once; with few tokens the heads are
    // shared among more warps.  (152 SMs of a GB300, with up to 32 warps each; nothing but this split depends on the number.)
    const int most = (heads + kHeads - 1) / kHeads;
    int64_t parts = ((int64_t)152 * 32 + a.n - 1) / a.n;
    parts = parts < 1 ? 1 : parts < most ? parts : most;
    a.part_heads = (int32_t)((most + parts - 1) / parts) * kHeads;
    a.parts = (heads + a.part_heads - 1) / a.part_heads;
    const int64_t warps = (int64_t)a.n * a.parts;
    const dim3 grid((unsigned)((warps + kRopeWarps - 1) / kRopeWarps));
    constexpr int kBlock = 32 * kRopeWarps;
    const bool norm = a.q_weight || a.k_weight;
    if (kind == kHalves)
        return norm ? kv4_launch(rope_kernel<D, T, kHalves, true, POOL>, grid, kBlock, 0, st, a)
                    : kv4_launch(rope_kernel<D, T, kHalves, false, POOL>, grid, kBlock, 0, st, a);
    if (kind == kNeighbours)
        return norm ? kv4_launch(rope_kernel<D, T, kNeighbours, true, POOL>, grid, kBlock, 0, st, a)
                    : kv4_launch(rope_kernel<D, T, kNeighbours, false, POOL>, grid, kBlock, 0, st, a);
    return norm ? kv4_launch(rope_kernel<D, T, kNoRotation, true, POOL>, grid, kBlock, 0, st, a)
                : kv4_launch(rope_kernel<D, T, kNoRotation, false, POOL>, grid, kBlock, 0, st, a);
}

template <bool POOL>
cudaError_t launch_rope(RopeArgs& a, int kind, int D, int dtype, cudaStream_t st)
{
    if (dtype == KVC_DTYPE_BF16) return D == 64 ? launch_rope<64, Bf16, POOL>(a, kind, st) : launch_rope<128, Bf16, POOL>(a, kind, st);
    return D == 64 ? launch_rope<64, Fp16, POOL>(a, kind, st) : launch_rope<128, Fp16, POOL>(a, kind, st);
}

int fail(const char* fn, int code, const char* what) noexcept
{
    try {
        return kv4_fail(code, (std::string(fn) + ": " + what).c_str());
    } catch (...) {
        return code;
    }
}

// What both entry points check; fills the arguments that they share.
int set_up(const char* fn, RopeArgs& a, const kv_rope* rope, int32_t head_dim, int32_t n, const int32_t* positions,
           int64_t axis_stride, int32_t hq, const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride,
           int32_t hkv, const void* k, int64_t k_stride, const void* q_weight, const void* k_weight, float eps,
           int* kind) noexcept
{
    if (n < 0) return fail(fn, KVC_ERR_INVALID, "n must be >= 0");
    if (hq < 0 || hq > 8192 || hkv < 0 || hkv > kKv4MaxHeads)
        return fail(fn, KVC_ERR_INVALID, "num_q_heads must be in 0 .. 8192, num_kv_heads in 0 .. 1024");
    *kind = kNoRotation;
    if (rope) {
        if (!rope->frequencies || !kv4_aligned(rope->frequencies, 8)) return fail(fn, KVC_ERR_INVALID, "kv_rope: frequencies must be an 8-byte aligned device pointer");
        if (rope->rotary_dim < 16 || rope->rotary_dim > head_dim || rope->rotary_dim % 16)
            return fail(fn, KVC_ERR_INVALID, "kv_rope: rotary_dim must be a multiple of 16 in 16 .. head_dim");
        if (rope->num_axes < 1 || rope->num_axes > 8) return fail(fn, KVC_ERR_INVALID, "kv_rope: num_axes must be in 1 .. 8");
        if (rope->neighbours != 0 && rope->neighbours != 1) return fail(fn, KVC_ERR_INVALID, "kv_rope: neighbours must be 0 or 1");
        if (!(rope->scale - rope->scale == 0.f)) return fail(fn, KVC_ERR_INVALID, "kv_rope: scale must be finite");
        if (n > 0 && (!positions || !kv4_aligned(positions, 4)))
            return fail(fn, KVC_ERR_INVALID, "positions must be a 4-byte aligned device pointer");
        if (axis_stride < 0) return fail(fn, KVC_ERR_INVALID, "axis_stride must be >= 0");
        *kind = rope->neighbours ? kNeighbours : kHalves;
        a.freqs = rope->frequencies;
        a.axes = rope->axes;
        a.num_axes = rope->num_axes;
        a.rot_chunks = rope->rotary_dim / 16;
        a.scale = rope->scale;
        a.positions = positions;
        a.axis_stride = axis_stride;
    }
    if ((q_weight && !kv4_aligned(q_weight, 16)) || (k_weight && !kv4_aligned(k_weight, 16)))
        return fail(fn, KVC_ERR_INVALID, "weights must be 16-byte aligned");
    if ((q_weight || k_weight) && !(eps >= 0x1p-100f && eps <= 0x1p100f))
        return fail(fn, KVC_ERR_INVALID, "eps must be in 2^-100 .. 2^100");
    if (n > 0 && hq > 0 && (!kv16_rows_ok(q, q_stride, n, 0, false) || !kv16_rows_ok(q_out, q_out_stride, n, (int64_t)hq * head_dim, true)))
        return fail(fn, KVC_ERR_INVALID, "q and q_out must be 16-byte aligned, their strides multiples of 8, q_out's rows apart");
    if (n > 0 && hkv > 0 && !kv16_rows_ok(k, k_stride, n, 0, false))
        return fail(fn, KVC_ERR_INVALID, "k must be 16-byte aligned, its stride a multiple of 8");
    a.eps = eps;
    a.n = n;
    a.hq = hq;
    a.hkv = hkv;
    a.q = static_cast<const uint16_t*>(q);
    a.q_out = static_cast<uint16_t*>(q_out);
    a.q_stride = q_stride;
    a.q_out_stride = q_out_stride;
    a.k = static_cast<const uint16_t*>(k);
    a.k_stride = k_stride;
    a.q_weight = static_cast<const uint16_t*>(q_weight);
    a.k_weight = static_cast<const uint16_t*>(k_weight);
    return KVC_OK;
}

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int kv_qk_rope(const kv_rope* rope, int32_t dtype, int32_t head_dim, int32_t n, const int32_t* positions,
                                  int64_t axis_stride, int32_t num_q_heads, const void* q, int64_t q_stride, void* q_out,
                                  int64_t q_out_stride, int32_t num_kv_heads, const void* k, int64_t k_stride, void* k_out,
                                  int64_t k_out_stride, const void* q_weight, const void* k_weight, float eps, void* stream)
{
    static const char fn[] = "kv_qk_rope";
    if (head_dim != 64 && head_dim != 128) return fail(fn, KVC_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (dtype != KVC_DTYPE_BF16 && dtype != KVC_DTYPE_F16) return fail(fn, KVC_ERR_INVALID, "unknown dtype");
    RopeArgs a{};
    int kind;
    if (int rc = set_up(fn, a, rope, head_dim, n, positions, axis_stride, num_q_heads, q, q_stride, q_out, q_out_stride,
                        num_kv_heads, k, k_stride, q_weight, k_weight, eps, &kind))
        return rc;
    if (n > 0 && num_kv_heads > 0 && !kv16_rows_ok(k_out, k_out_stride, n, (int64_t)num_kv_heads * head_dim, true))
        return fail(fn, KVC_ERR_INVALID, "k_out must be 16-byte aligned, its stride a multiple of 8, its rows apart");
    if (n == 0 || num_q_heads + num_kv_heads == 0) return KVC_OK;
    a.k_out = static_cast<uint16_t*>(k_out);
    a.k_out_stride = k_out_stride;
    return kv4_launch_result(launch_rope<false>(a, kind, head_dim, dtype, static_cast<cudaStream_t>(stream)));
}

extern "C" KVC_API int kv16_write(const kv16_pool* pool, const kv_rope* rope, int32_t n, const int64_t* slots,
                                  const int32_t* positions, int64_t axis_stride, int32_t num_q_heads, const void* q,
                                  int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride,
                                  const void* v, int64_t v_stride, const void* q_weight, const void* k_weight, float eps,
                                  int32_t* device_error, void* stream)
{
    static const char fn[] = "kv16_write";
    if (int rc = kv16_check_pool(pool, true)) return rc;
    RopeArgs a{};
    int kind;
    if (int rc = set_up(fn, a, rope, pool->head_dim, n, positions, axis_stride, num_q_heads, q, q_stride, q_out, q_out_stride,
                        pool->num_kv_heads, k, k_stride, q_weight, k_weight, eps, &kind))
        return rc;
    if (n > 0 && (!slots || !kv4_aligned(slots, 8))) return fail(fn, KVC_ERR_INVALID, "slots must be an 8-byte aligned device pointer");
    if (n > 0 && !kv16_rows_ok(v, v_stride, n, 0, false))
        return fail(fn, KVC_ERR_INVALID, "v must be 16-byte aligned, its stride a multiple of 8");
    if (n == 0) return KVC_OK;
    a.v = static_cast<const uint16_t*>(v);
    a.v_stride = v_stride;
    a.k_out = static_cast<uint16_t*>(pool->k);
    a.v_out = static_cast<uint16_t*>(pool->v);
    a.slots = slots;
    a.num_slots = pool->num_pages * kPageSize;
    a.err = device_error;
    return kv4_launch_result(launch_rope<true>(a, kind, pool->head_dim, pool->dtype, static_cast<cudaStream_t>(stream)));
}
