// Shared by the translation units of the 16-bit serving step (kvdecode16.h):
// argument checks.  Not part of the ABI.
#pragma once

#include "kvd_kv4.h"
#include "kvdecode16.h"

namespace kvd {

constexpr int kKv16MaxBatch = 4096;

inline int kv16_check_pool(const kv16_pool* p, bool data) noexcept
{
    if (!p) return kv4_fail(KVC_ERR_INVALID, "kv16_pool: null pool");
    if (p->head_dim != 64 && p->head_dim != 128) return kv4_fail(KVC_ERR_UNSUPPORTED, "kv16_pool: head_dim must be 64 or 128");
    if (p->dtype != KVC_DTYPE_BF16 && p->dtype != KVC_DTYPE_F16) return kv4_fail(KVC_ERR_INVALID, "kv16_pool: unknown dtype");
    if (p->num_kv_heads < 1 || p->num_kv_heads > kKv4MaxHeads)
        return kv4_fail(KVC_ERR_INVALID, "kv16_pool: num_kv_heads must be in 1 .. 1024");
    if (p->num_pages < 1 || p->num_pages >= (int64_t)1 << 27 || p->num_pages * p->num_kv_heads >= (int64_t)1 << 27)
        return kv4_fail(KVC_ERR_INVALID, "kv16_pool: num_pages must be >= 1, num_pages * num_kv_heads below 2^27");
    if (data && (!p->k || !p->v || !kv4_aligned(p->k, 16) || !kv4_aligned(p->v, 16)))
        return kv4_fail(KVC_ERR_INVALID, "kv16_pool: k and v must be 16-byte aligned device pointers");
    return KVC_OK;
}

// Rows [n][heads][d] that a call reads or writes.
inline bool kv16_rows_ok(const void* p, int64_t stride, int32_t n, int64_t width, bool out)
{
    return p && kv4_aligned(p, 16) && stride % 8 == 0 && (n <= 1 ? stride >= 0 : out ? stride >= width : stride >= 0);
}

inline int kv16_check_heads(const kv16_pool* pool, int32_t hq, int32_t batch) noexcept
{
    if (int rc = kv16_check_pool(pool, false)) return rc;
    if (batch < 1 || batch > kKv16MaxBatch) return kv4_fail(KVC_ERR_INVALID, "kv16: the batch must be in 1 .. 4096");
    if (hq < 1 || hq % pool->num_kv_heads) return kv4_fail(KVC_ERR_INVALID, "kv16: num_q_heads must be a multiple of num_kv_heads");
    if (hq / pool->num_kv_heads > 8) return kv4_fail(KVC_ERR_UNSUPPORTED, "kv16: more than 8 query heads per KV head");
    return KVC_OK;
}

inline int kv16_sms(int* sms) noexcept
{
    int device = 0;
    if (cudaError_t e = cudaGetDevice(&device); e != cudaSuccess) return kv4_launch_result(e);
    return kv4_launch_result(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
}

}  // namespace kvd
