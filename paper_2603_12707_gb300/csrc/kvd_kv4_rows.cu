// kv4_write and kv4_read: K and V rows of tokens into and out of the 4-bit
// pool's blocks (layout and quantisation: kvdecode4.h).
//
// One warp per (token, KV head, K or V).  A lane holds D / 32 consecutive
// elements, a scale group lies in group * 32 / D lanes, and the codes pass
// through a row of shared memory into the words of the block.
#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kRowWarps = 8;

struct RowsArgs {
    uint8_t* pool;
    int64_t num_slots;     // num_pages * 16
    int32_t H, n;
    const int64_t* slots;
    uint16_t* k;           // [n][H][D], row strides k_stride and v_stride
    uint16_t* v;
    int64_t k_stride, v_stride;
    int32_t* err;
};

template <int D, int NG>
struct RowPlace {   // where a token's row lies in its block
    uint8_t* codes;
    uint32_t* scales;
    int tok;
    __device__ __forceinline__ RowPlace(uint8_t* pool, int64_t slot, int H, int h, bool is_v)
    {
        using B = Kv4Block<D, NG>;
        tok = (int)(slot & (kPageSize - 1));
        uint8_t* block = pool + ((slot >> 4) * H + h) * B::kBytes;
        codes = block + (is_v ? B::kCodes : 0);
        scales = reinterpret_cast<uint32_t*>(block + 2 * B::kCodes + (is_v ? B::kScales : 0)) + tok * NG;
    }
};

// K word m of a token: [j][i]; V half-word m: [g][i].
template <int D>
__device__ __forceinline__ int k_element(int m, int e)
{
    constexpr int NW = D / 32;
    return 32 * (m % NW) + 8 * (m / NW) + e;
}
template <int D>
__device__ __forceinline__ int v_element(int m, int n)
{
    constexpr int NW = D / 32;
    return 32 * (m % NW) + 8 * n + m / NW;
}
template <int D>
__device__ __forceinline__ int v_half_offset(int tok, int m)   // bytes from the V codes' start
{
    constexpr int NW = D / 32;
    const int g = m / NW, i = m % NW;
    return ((((tok >> 3) * 8 + g) * 4 + ((tok & 7) >> 1)) * NW + i) * 4 + (tok & 1) * 2;
}

template <int D, int NG, class T>
__global__ void __launch_bounds__(kRowWarps * 32) write_kernel(RowsArgs a)
{
    constexpr int E = D / 32;              // elements of a lane
    constexpr int GL = 32 / NG;            // lanes of a group
    __shared__ uint8_t row[kRowWarps][D];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t rows = (int64_t)a.n * a.H * 2;
    for (int64_t r = (int64_t)blockIdx.x * kRowWarps + warp; r < rows; r += (int64_t)gridDim.x * kRowWarps) {
        const bool is_v = r & 1;
        const int h = (int)((r >> 1) % a.H);
        const int64_t tok = (r >> 1) / a.H;
        const int64_t slot = a.slots[tok];
        if (slot < 0 || slot >= a.num_slots) {
            if (slot != -1 && lane == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
            continue;
        }
        const uint16_t* src = (is_v ? a.v + tok * a.v_stride : a.k + tok * a.k_stride) + (int64_t)h * D + lane * E;
        uint32_t w[E / 2];
        if constexpr (E == 4) {
            const uint2 u = *reinterpret_cast<const uint2*>(src);
            w[0] = u.x;
            w[1] = u.y;
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(src);
        }
        float x[E];
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            x[2 * i] = T::lo(w[i]);
            x[2 * i + 1] = T::hi(w[i]);
        }
        float lo = x[0], hi = x[0], sum = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            lo = fminf(lo, x[i]);
            hi = fmaxf(hi, x[i]);
            sum += x[i] * 0.f;             // NaN where an element is not finite
        }
#pragma unroll
        for (int m = 1; m < GL; m <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, m));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, m));
            sum += __shfl_xor_sync(0xffffffffu, sum, m);
        }
        // s and z as they are held; the codes follow from those.
        uint32_t meta = T::pack((hi * 0.5f - lo * 0.5f) / 7.5f, 0.f);
        float s = T::lo(meta);
        meta = (meta & 0xffffu) | (T::pack(fmaf(8.f, s, lo), 0.f) << 16);
        float z = T::hi(meta);
        if (sum != 0.f) meta = T::pack(__int_as_float(0x7fc00000), __int_as_float(0x7fc00000));
        const bool flat = !(s > 0.f) || sum != 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float c = flat ? 8.f : fminf(fmaxf(rintf((x[i] - z) / s) + 8.f, 0.f), 15.f);
            row[warp][lane * E + i] = (uint8_t)(int)c;
        }
        __syncwarp();
        const RowPlace<D, NG> to(a.pool, slot, a.H, h, is_v);
        if (lane % GL == 0) to.scales[lane / GL] = meta;
        if (!is_v) {
            if (lane < D / 8) {
                uint32_t word = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) word |= (uint32_t)row[warp][k_element<D>(lane, e)] << (16 * (e & 1) + 4 * (e >> 1));
                reinterpret_cast<uint32_t*>(to.codes)[to.tok * (D / 8) + lane] = word;
            }
        } else if (lane < D / 4) {
            uint32_t half = 0;
#pragma unroll
            for (int n = 0; n < 4; ++n) half |= (uint32_t)row[warp][v_element<D>(lane, n)] << (4 * n);
            *reinterpret_cast<uint16_t*>(to.codes + v_half_offset<D>(to.tok, lane)) = (uint16_t)half;
        }
        __syncwarp();
    }
}

template <int D, int NG, class T>
__global__ void __launch_bounds__(kRowWarps * 32) read_kernel(RowsArgs a)
{
    constexpr int E = D / 32;
    constexpr int GL = 32 / NG;
    __shared__ uint8_t row[kRowWarps][D];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t rows = (int64_t)a.n * a.H * 2;
    for (int64_t r = (int64_t)blockIdx.x * kRowWarps + warp; r < rows; r += (int64_t)gridDim.x * kRowWarps) {
        const bool is_v = r & 1;
        const int h = (int)((r >> 1) % a.H);
        const int64_t tok = (r >> 1) / a.H;
        const int64_t slot = a.slots[tok];
        uint16_t* dst = (is_v ? a.v + tok * a.v_stride : a.k + tok * a.k_stride) + (int64_t)h * D + lane * E;
        uint32_t w[E / 2] = {};
        if (slot >= 0 && slot < a.num_slots) {
            const RowPlace<D, NG> from(a.pool, slot, a.H, h, is_v);
            if (!is_v) {
                if (lane < D / 8) {
                    const uint32_t word = reinterpret_cast<const uint32_t*>(from.codes)[from.tok * (D / 8) + lane];
#pragma unroll
                    for (int e = 0; e < 8; ++e) row[warp][k_element<D>(lane, e)] = (word >> (16 * (e & 1) + 4 * (e >> 1))) & 15;
                }
            } else if (lane < D / 4) {
                const uint32_t half = *reinterpret_cast<const uint16_t*>(from.codes + v_half_offset<D>(from.tok, lane));
#pragma unroll
                for (int n = 0; n < 4; ++n) row[warp][v_element<D>(lane, n)] = (half >> (4 * n)) & 15;
            }
            __syncwarp();
            const uint32_t meta = from.scales[lane / GL];
            const float s = T::lo(meta), z = T::hi(meta);
            float x[E];
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = fmaf(s, (float)row[warp][lane * E + i] - 8.f, z);
#pragma unroll
            for (int i = 0; i < E / 2; ++i) w[i] = T::pack(x[2 * i], x[2 * i + 1]);
            __syncwarp();
        } else if (slot != -1 && lane == 0) {
            kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
        }
        if constexpr (E == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(dst) = w[0];
    }
}

template <bool kWrite>
struct LaunchRows {
    const RowsArgs& a;
    cudaStream_t st;
    template <int D, int NG, class T>
    cudaError_t operator()() const
    {
        const int64_t rows = (int64_t)a.n * a.H * 2;
        const int64_t ctas = (rows + kRowWarps - 1) / kRowWarps;
        const dim3 grid((unsigned)(ctas < (1 << 20) ? ctas : (1 << 20)));
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
