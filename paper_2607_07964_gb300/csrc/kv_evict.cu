// kq_kv_evict: one block for a sequence and head. The threshold is found bit by bit (the largest
// key that `budget` slots reach), slots equal to it are taken from the lowest on, and the kept slots
// past the budget move into the free ones before it through two lists in the workspace.
#include <algorithm>

#include "kv_common.cuh"

namespace kq {
namespace {

constexpr int kThreads = 1024;

// Order-preserving key of a slot: protected above every weight, NaN below.
__device__ __forceinline__ uint32_t evict_key(float w, int64_t pos, int64_t from, int64_t sink) {
    if (pos >= from || pos < sink) return 0xFFFFFFFFu;
    if (isnan(w)) return 0u;
    const uint32_t u = __float_as_uint(w == 0.0f ? 0.0f : w);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

// Exclusive prefix sum of v over the block; total receives the sum.
__device__ __forceinline__ int block_scan(int v, int* tmp, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) tmp[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int y = tmp[lane];
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) y += u;
        }
        tmp[lane] = y;
    }
    __syncthreads();
    total = tmp[31];
    return x - v + (warp ? tmp[warp - 1] : 0);
}

__global__ void __launch_bounds__(kThreads) kv_evict_kernel(KvView c, const int32_t* __restrict__ lens, const float* acc,
                                                            const int32_t* pos, const int32_t* __restrict__ seen, int64_t S,
                                                            int64_t budget, int64_t recent, int64_t sink, int32_t* lens_out,
                                                            float* acc_out, int32_t* pos_out, int32_t* __restrict__ lists,
                                                            int* info) {
    __shared__ int tmp[32];
    const int b = blockIdx.x / c.kv_heads, h = blockIdx.x % c.kv_heads, tid = threadIdx.x;
    const int64_t n = kv_length(lens, b, min(kv_capacity(c), S), info);
    if (h == 0 && tid == 0) lens_out[b] = static_cast<int32_t>(min(n, budget));
    const int64_t row = static_cast<int64_t>(blockIdx.x) * S;
    acc += row, pos += row, acc_out += row, pos_out += row;
    if (n <= budget) {
        for (int64_t j = tid; j < n; j += kThreads) acc_out[j] = acc[j], pos_out[j] = pos[j];
        return;
    }
    const int64_t from = static_cast<int64_t>(seen[b]) - recent;
    uint32_t t = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t cand = t | (1u << bit);
        int mine = 0, all;
        for (int64_t j = tid; j < n; j += kThreads) mine += evict_key(acc[j], pos[j], from, sink) >= cand;
        block_scan(mine, tmp, all);
        if (all >= budget) t = cand;
    }
    int mine = 0, above;
    for (int64_t j = tid; j < n; j += kThreads) mine += evict_key(acc[j], pos[j], from, sink) > t;
    block_scan(mine, tmp, above);
    const int64_t quota = budget - above;   // slots equal to the threshold that are kept
    int32_t* hole = lists + static_cast<int64_t>(blockIdx.x) * 2 * budget;
    int32_t* tail = hole + budget;
    int64_t ties = 0, holes = 0, tails = 0;
    for (int64_t base = 0; base < n; base += kThreads) {
        const int64_t j = base + tid;
        uint32_t key = 0;
        if (j < n) key = evict_key(acc[j], pos[j], from, sink);
        const int eq = j < n && key == t;
        int all;
        const int64_t before = ties + block_scan(eq, tmp, all);
        ties += all;
        const bool keep = j < n && (key > t || (eq && before < quota));
        const int is_hole = j < budget && !keep, is_tail = j >= budget && keep;
        int at = block_scan(is_hole, tmp, all);
        if (is_hole) hole[holes + at] = static_cast<int32_t>(j);
        holes += all;
        at = block_scan(is_tail, tmp, all);
        if (is_tail) tail[tails + at] = static_cast<int32_t>(j);
        tails += all;
    }
    __syncthreads();
    if (acc_out != acc)
        for (int64_t j = tid; j < budget; j += kThreads) acc_out[j] = acc[j];
    if (pos_out != pos)
        for (int64_t j = tid; j < budget; j += kThreads) pos_out[j] = pos[j];
    __syncthreads();
    for (int64_t m = tid >> 5; m < holes; m += kThreads / 32) {
        const int64_t to = hole[m], at = tail[m];
        const uint8_t* src = kv_granule(c, b, h, at);
        uint8_t* dst = kv_granule(c, b, h, to);
        if (!src || !dst) {
            record_error(info, -KQ_ERR_INVALID_ARG);
            continue;
        }
        const int lane = tid & 31, ts = static_cast<int>(at % kGranule), td = static_cast<int>(to % kGranule);
        for (int which = 0; which < 2; ++which) {
            if (lane < c.dim / 8)
                reinterpret_cast<uint32_t*>(dst + kv_code_at(c.dim, which, td))[lane] =
                    reinterpret_cast<const uint32_t*>(src + kv_code_at(c.dim, which, ts))[lane];
            if (lane == 31)
                *reinterpret_cast<uint32_t*>(dst + kv_param_at(c.dim, which, td)) =
                    *reinterpret_cast<const uint32_t*>(src + kv_param_at(c.dim, which, ts));
        }
        if (lane == 30) acc_out[to] = acc[at], pos_out[to] = pos[at];
    }
}

}  // namespace

KQ_DEBUG_UNIT(kv_evict)
}  // namespace kq

using namespace kq;

extern "C" size_t kq_kv_evict_workspace(int64_t batch, int64_t kv_heads, int64_t S, int64_t budget) {
    if (batch < 1 || kv_heads < 1 || S < 1 || budget < 1) return 0;
    return static_cast<size_t>(batch) * kv_heads * 2 * std::min(budget, S) * sizeof(int32_t);
}

extern "C" kq_status kq_kv_evict(const kq_kv_cache* cache, const int32_t* lens, const float* acc, const int32_t* pos,
                                 const int32_t* seen, int64_t S, int64_t budget, int64_t recent, int64_t sink,
                                 int32_t* lens_out, float* acc_out, int32_t* pos_out, int* info, void* ws,
                                 size_t ws_bytes, kq_stream_t stream_) {
    KvView c;
    KQ_TRY(kv_view(cache, "kq_kv_evict", &c));
    if (!lens || !acc || !pos || !seen || !lens_out || !acc_out || !pos_out || lens_out == lens || S < 1 ||
        S > 0x7fffffffll || budget < 1 || recent < 0 || sink < 0 || recent > budget || sink > budget - recent) {
        set_error("kq_kv_evict: arrays must not be NULL, lens_out apart from lens, budget >= 1, recent + sink <= budget");
        return KQ_ERR_INVALID_ARG;
    }
    budget = std::min(budget, S);
    const size_t need = kq_kv_evict_workspace(c.batch, c.kv_heads, S, budget);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("kq_kv_evict: workspace must be 256-byte aligned and hold %zu bytes", need);
        return KQ_ERR_WORKSPACE;
    }
    kv_evict_kernel<<<static_cast<unsigned>(c.batch * c.kv_heads), kThreads, 0, reinterpret_cast<cudaStream_t>(stream_)>>>(
        c, lens, acc, pos, seen, S, budget, recent, sink, lens_out, acc_out, pos_out, static_cast<int32_t*>(ws), info);
    KQ_LAUNCH_CHECK("kv_evict_kernel");
    return KQ_OK;
}
