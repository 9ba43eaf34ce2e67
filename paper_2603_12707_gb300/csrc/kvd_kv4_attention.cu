// kv4_decode_attention: single-token decode attention over the 4-bit paged
// cache (layout: kvdecode4.h).
//
// One CTA per (row, KV head).  Its warps take tokens in turn; each keeps a
// running maximum, sum and output (an online softmax) for the G query heads of
// the KV head, and the warps' results are merged in shared memory.
#include <cmath>

#include "kvd_kv4.h"
#include "kvd_ptx.cuh"

namespace kvd {
namespace {

constexpr int kAttnWarps = 4;

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
    float scale_log2;
    int32_t* err;
};

template <int D, int NG, class T>
__global__ void __launch_bounds__(kAttnWarps * 32) attention_kernel(AttnArgs a)
{
    using B = Kv4Block<D, NG>;
    constexpr int E = D / 32, NW = D / 32, GL = 32 / NG;
    __shared__ float so[kAttnWarps][kMaxGroup][D];
    __shared__ float sm[kAttnWarps][kMaxGroup], sl[kAttnWarps][kMaxGroup];
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int b = blockIdx.x / a.H, h = blockIdx.x % a.H;
    const int seq = a.seq_ids ? a.seq_ids[b] : b;
    int len = seq >= 0 && seq < a.max_seqs ? a.lens[seq] : -1;
    if (len < 0 || len > (int64_t)a.max_pages * kPageSize) {
        if (threadIdx.x == 0) kv4_error(a.err, KVC_DEVERR_SEQ_RANGE);
        len = 0;
    }
    float q[kMaxGroup][E], o[kMaxGroup][E], m[kMaxGroup], l[kMaxGroup];
    for (int n = 0; n < kMaxGroup; ++n) {
        m[n] = -INFINITY;
        l[n] = 0.f;
        for (int i = 0; i < E; ++i) {
            o[n][i] = 0.f;
            const uint16_t x = n < a.G ? a.q[b * a.q_stride + (int64_t)(h * a.G + n) * D + lane * E + i] : 0;
            q[n][i] = T::lo(x) * a.scale_log2;
        }
    }
    for (int t = warp; t < len; t += kAttnWarps) {
        const int32_t page = a.block_table[(int64_t)seq * a.max_pages + t / kPageSize];
        if (page < 0 || page >= a.num_pages) {
            if (lane == 0) kv4_error(a.err, KVC_DEVERR_PAGE_RANGE);
            continue;
        }
        const uint8_t* block = a.pool + ((int64_t)page * a.H + h) * B::kBytes;
        const int s = t % kPageSize;
        const uint32_t* scales = reinterpret_cast<const uint32_t*>(block + 2 * B::kCodes) + s * NG + lane / GL;
        const uint32_t mk = scales[0], mv = scales[kPageSize * NG];
        float k[E], v[E];
        for (int i = 0; i < E; ++i) {
            const int d = lane * E + i, e = d % 8, j = (d / 8) % 4, w = d / 32;
            const uint32_t kw = reinterpret_cast<const uint32_t*>(block)[(s * 4 + j) * NW + w];
            k[i] = T::lo(mk) * ((float)((kw >> (16 * (e & 1) + 4 * (e >> 1))) & 15) - 8.f) + T::hi(mk);
            const uint32_t vw = reinterpret_cast<const uint32_t*>(block + B::kCodes)[((s / 8 * 8 + e) * 4 + (s % 8) / 2) * NW + w];
            v[i] = T::lo(mv) * ((float)((vw >> (16 * (s & 1) + 4 * j)) & 15) - 8.f) + T::hi(mv);
        }
#pragma unroll
        for (int n = 0; n < kMaxGroup; ++n) {
            if (n >= a.G) break;
            float x = 0.f;
            for (int i = 0; i < E; ++i) x += q[n][i] * k[i];
            for (int mask = 1; mask < 32; mask <<= 1) x += __shfl_xor_sync(0xffffffffu, x, mask);
            const float top = fmaxf(m[n], x), al = exp2f(m[n] - top), p = exp2f(x - top);
            m[n] = top;
            l[n] = l[n] * al + p;
            for (int i = 0; i < E; ++i) o[n][i] = o[n][i] * al + p * v[i];
        }
    }
    for (int n = 0; n < kMaxGroup; ++n) {
        for (int i = 0; i < E; ++i) so[warp][n][lane * E + i] = o[n][i];
        if (lane == 0) {
            sm[warp][n] = m[n];
            sl[warp][n] = l[n];
        }
    }
    __syncthreads();
    for (int n = warp; n < a.G; n += kAttnWarps) {
        float top = -INFINITY, sum = 0.f, x[E] = {};
        for (int w = 0; w < kAttnWarps; ++w) top = fmaxf(top, sm[w][n]);
        for (int w = 0; w < kAttnWarps; ++w) {
            const float al = sl[w][n] == 0.f ? 0.f : exp2f(sm[w][n] - top);
            sum += al * sl[w][n];
            for (int i = 0; i < E; ++i) x[i] += al * so[w][n][lane * E + i];
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint16_t* out = a.out + b * a.out_stride + (int64_t)(h * a.G + n) * D + lane * E;
        for (int i = 0; i < E; ++i) out[i] = (uint16_t)T::pack(x[i] * inv, 0.f);
        if (a.lse && lane == 0) a.lse[(int64_t)b * a.Hq + h * a.G + n] = (top + log2f(sum)) * 0.6931471805599453f;
    }
}

struct LaunchAttention {
    const AttnArgs& a;
    cudaStream_t st;
    template <int D, int NG, class T>
    cudaError_t operator()() const
    {
        return kv4_launch(attention_kernel<D, NG, T>, dim3((unsigned)(a.batch * a.H)), kAttnWarps * 32, 0, st, a);
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

int64_t workspace_bytes_of(const kv4_pool&, int32_t) { return 256; }

}  // namespace
}  // namespace kvd

using namespace kvd;

extern "C" KVC_API int64_t kv4_workspace_bytes(const kv4_pool* pool, int32_t num_q_heads)
{
    if (int rc = kv4_check_pool(pool, false)) return rc;
    if (int rc = check_heads(pool, num_q_heads)) return rc;
    return workspace_bytes_of(*pool, num_q_heads);
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
    if (!kv4_aligned(workspace, 256) || workspace_bytes < workspace_bytes_of(*pool, num_q_heads))
        return kv4_fail(KVC_ERR_INVALID, "kv4_decode_attention: workspace must be 256-byte aligned and of kv4_workspace_bytes()");
    const float scale = softmax_scale > 0.f ? softmax_scale : 1.0f / std::sqrt((float)pool->head_dim);
    AttnArgs a{};
    a.pool = static_cast<const uint8_t*>(pool->data);
    a.num_pages = pool->num_pages;
    a.H = pool->num_kv_heads;
    a.Hq = num_q_heads;
    a.G = num_q_heads / pool->num_kv_heads;
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
    a.scale_log2 = scale * 1.4426950408889634f;
    a.err = device_error;
    return kv4_launch_result(kv4_dispatch(*pool, LaunchAttention{a, static_cast<cudaStream_t>(stream)}));
}
