// Shared by the translation units of the 4-bit cache (kvdecode4.h): argument
// checks, launches, and the layout of a pool's blocks.  Not part of the ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kvd_internal.h"
#include "kvd_ptx.cuh"
#include "kvdecode4.h"

namespace kvd {

constexpr int kKv4MaxBatch = 4096;
constexpr int kKv4MaxHeads = 1024;

// A failed call's code, with its message for kv_last_error().
inline int kv4_fail(int code, const char* msg) noexcept
{
    try {
        set_last_error(msg);
    } catch (...) {   // no memory for the message: the code still says what happened
    }
    return code;
}

inline int kv4_launch_result(cudaError_t e) noexcept
{
    return e == cudaSuccess ? KVC_OK : kv4_fail(KVC_ERR_CUDA, cudaGetErrorString(e));
}

inline bool kv4_aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// KVC_OK, or why the pool's description is refused.
inline int kv4_check_pool(const kv4_pool* p, bool data) noexcept
{
    if (!p) return kv4_fail(KVC_ERR_INVALID, "kv4_pool: null pool");
    if (p->head_dim != 64 && p->head_dim != 128) return kv4_fail(KVC_ERR_UNSUPPORTED, "kv4_pool: head_dim must be 64 or 128");
    if (p->group != 32 && p->group != 64 && p->group != p->head_dim)
        return kv4_fail(KVC_ERR_UNSUPPORTED, "kv4_pool: group must be 32, 64 or head_dim");
    if (p->dtype != KVC_DTYPE_BF16 && p->dtype != KVC_DTYPE_F16) return kv4_fail(KVC_ERR_INVALID, "kv4_pool: unknown dtype");
    if (p->num_kv_heads < 1 || p->num_kv_heads > kKv4MaxHeads)
        return kv4_fail(KVC_ERR_INVALID, "kv4_pool: num_kv_heads must be in 1 .. 1024");
    if (p->num_pages < 1 || p->num_pages >= (int64_t)1 << 31)
        return kv4_fail(KVC_ERR_INVALID, "kv4_pool: num_pages must be in 1 .. 2^31 - 1");
    if (data && (!p->data || !kv4_aligned(p->data, 128)))
        return kv4_fail(KVC_ERR_INVALID, "kv4_pool: data must be a 128-byte aligned device pointer");
    return KVC_OK;
}

inline int kv4_check_tables(const kv_tables* t) noexcept
{
    if (!t || !t->block_table || !t->lens) return kv4_fail(KVC_ERR_INVALID, "kv_tables: null argument");
    if (t->max_seqs < 1 || t->max_pages < 1 || (int64_t)t->max_seqs * t->max_pages >= (int64_t)1 << 31)
        return kv4_fail(KVC_ERR_INVALID, "kv_tables: max_seqs and max_pages must be >= 1 with a product below 2^31");
    if ((int64_t)t->max_pages * kPageSize >= (int64_t)1 << 31)
        return kv4_fail(KVC_ERR_INVALID, "kv_tables: max_pages * 16 must be below 2^31");
    return KVC_OK;
}

// Layout of the block of one (page, KV head).
template <int D, int NG>   // NG: scale groups of a token's row
struct Kv4Block {
    static constexpr int kCodes = kPageSize * D / 2;          // bytes of K's codes, and of V's
    static constexpr int kScales = kPageSize * NG * 4;        // bytes of K's scales, and of V's
    static constexpr int kBytes = 2 * (kCodes + kScales);
};

__host__ inline int64_t kv4_block_bytes(const kv4_pool& p) { return 16 * p.head_dim + 128 * (p.head_dim / p.group); }

// The cache's 16-bit type.
struct Bf16 {
    static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_bf16(a, b); }
    static __device__ __forceinline__ uint32_t pack_finite(float a, float b)   // (what rounds to an infinity: the largest number)
    {
        uint32_t r;
        asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
        return r;
    }
    static __device__ __forceinline__ uint32_t toward_zero(float a) { return __float_as_uint(a) >> 16; }
    static constexpr float kOver = 0x1.ffp127f, kNear = 0x1.f0p127f;   // the least that rounds to infinity; groups below kNear hold nothing that does
};
struct Fp16 {
    static __device__ __forceinline__ float lo(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xffffu))); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { return pack_f16(a, b); }
    static __device__ __forceinline__ uint32_t pack_finite(float a, float b)
    {
        uint32_t r;
        asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
        return r;
    }
    static __device__ __forceinline__ uint32_t toward_zero(float a) { return __half_as_ushort(__float2half_rz(a)); }
    static constexpr float kOver = 65520.f, kNear = 65300.f;
};

__device__ __forceinline__ void kv4_error(int32_t* err, int32_t bit)
{
    if (err) atomicOr(err, bit);
}

// A launch that may be placed before the one before it has completed; the
// kernel waits for that first (griddep_wait).
template <class... P, class... A>
inline cudaError_t kv4_launch(void (*kernel)(P...), dim3 grid, int block, size_t smem, cudaStream_t st, const A&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Calls f with the pool's shape and type as template parameters:
// f.template operator()<D, NG, T>().
template <class F>
inline auto kv4_dispatch(const kv4_pool& p, F&& f)
{
    const int ng = p.head_dim / p.group;
    if (p.dtype == KVC_DTYPE_BF16) {
        if (p.head_dim == 64) return ng == 1 ? f.template operator()<64, 1, Bf16>() : f.template operator()<64, 2, Bf16>();
        return ng == 1   ? f.template operator()<128, 1, Bf16>()
               : ng == 2 ? f.template operator()<128, 2, Bf16>()
                         : f.template operator()<128, 4, Bf16>();
    }
    if (p.head_dim == 64) return ng == 1 ? f.template operator()<64, 1, Fp16>() : f.template operator()<64, 2, Fp16>();
    return ng == 1   ? f.template operator()<128, 1, Fp16>()
           : ng == 2 ? f.template operator()<128, 2, Fp16>()
                     : f.template operator()<128, 4, Fp16>();
}

}  // namespace kvd
