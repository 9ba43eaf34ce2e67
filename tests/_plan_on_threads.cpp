// plan_kernel on host threads, one for each of a CTA's, CTAs one after another.  The kernel's source is compiled as it is: PLAN_SOURCE is
// kvd_kv16_plan.h and kvd_kv16_plan.cu up to its entry point, without their includes.
#include <pthread.h>

#include <chrono>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <memory>
#include <thread>
#include <vector>

#include "kvdecode16.h"

#define __host__
#define __device__
#define __global__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define __restrict__

struct float2 { float x, y; };
struct Dim { int x; };
static thread_local Dim threadIdx, blockIdx;
static Dim blockDim, gridDim;
static int64_t shared_memory[1 << 15];
struct Barrier {
    pthread_barrier_t b;
    explicit Barrier(int n) { pthread_barrier_init(&b, nullptr, n); }
    ~Barrier() { pthread_barrier_destroy(&b); }
    void wait() { pthread_barrier_wait(&b); }
};
static std::unique_ptr<Barrier> cta_barrier;
static std::vector<std::unique_ptr<Barrier>> warp_barriers, pair_barriers;
static uint64_t exchange[16][32];
static int late;      // 0: nobody; 1: all warps but the first dawdle after a barrier of the CTA; 2: the first does

static void __syncthreads()
{
    cta_barrier->wait();
    const bool first = threadIdx.x < 32;
    if ((late == 1 && !first) || (late == 2 && first)) std::this_thread::sleep_for(std::chrono::milliseconds(3));
}
static void __syncwarp(uint32_t mask) { (mask == 3u ? pair_barriers : warp_barriers)[threadIdx.x >> 5]->wait(); }
template <class V>
static V shuffle(V v, int from)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    std::memcpy(&exchange[warp][lane], &v, sizeof v);
    warp_barriers[warp]->wait();
    if (from >= 0) std::memcpy(&v, &exchange[warp][from], sizeof v);
    warp_barriers[warp]->wait();
    return v;
}
template <class V>
static V __shfl_up_sync(uint32_t, V v, int n) { return shuffle(v, (int)(threadIdx.x & 31) - n); }
template <class V>
static V __shfl_sync(uint32_t, V v, int from) { return shuffle(v, from); }
static float __fdividef(float a, float b) { return a / b; }
static int min(int a, int b) { return a < b ? a : b; }
static int max(int a, int b) { return a > b ? a : b; }
static int64_t min(int64_t a, int64_t b) { return a < b ? a : b; }
static float max(float a, float b) { return a > b ? a : b; }

namespace kvd {
constexpr int kPageSize = 16;
static void griddep_wait() {}
static void griddep_launch_dependents() {}
static void kv4_error(int32_t* err, int32_t bit) { __atomic_fetch_or(err, bit, __ATOMIC_RELAXED); }
}  // namespace kvd

#include PLAN_SOURCE

using namespace kvd;
static_assert(sizeof(PlanHeader) == 72 && sizeof(Record) == 32 && sizeof(Run) == 32 && sizeof(RowSources) == 32 && sizeof(WarpStart) == 64 &&
                  sizeof(CtaStart) == 88,
              "what _kv16_plan.py reads");

// As kv16_plan launches it, with `ctas` CTAs of `threads`; CTA c dawdles as `dawdle[c]` says.
extern "C" int64_t plan(const int32_t* lens, const int32_t* seq_ids, const int32_t* prefix_ids, int max_seqs, int max_pages, int batch, int hq,
                        int hkv, int dim, int grid, int threads, int ctas, const int32_t* dawdle, void* workspace, int32_t* err)
{
    StepPlanArgs a{};
    a.view = plan_view(workspace, batch, hq, hkv, dim, grid);
    if (!workspace) return a.view.bytes;
    a.lens = lens;
    a.seq_ids = seq_ids;
    a.prefix_ids = prefix_ids;
    a.max_seqs = max_seqs;
    a.max_pages = max_pages;
    a.batch = batch;
    a.hq = hq;
    a.hkv = hkv;
    a.dim = dim;
    a.grid = grid;
    a.err = err;
    blockDim.x = threads;
    gridDim.x = ctas;
    cta_barrier = std::make_unique<Barrier>(threads);
    warp_barriers.clear();
    pair_barriers.clear();
    for (int w = 0; w < threads / 32; ++w) {
        warp_barriers.push_back(std::make_unique<Barrier>(32));
        pair_barriers.push_back(std::make_unique<Barrier>(2));
    }
    for (int c = 0; c < ctas; ++c) {
        late = dawdle[c];
        std::memset(shared_memory, 0xa5, sizeof shared_memory);
        std::vector<std::thread> all;
        for (int t = 0; t < threads; ++t)
            all.emplace_back([&, t] {
                threadIdx.x = t;
                blockIdx.x = c;
                plan_kernel(a);
            });
        for (auto& t : all) t.join();
    }
    return a.view.bytes;
}
