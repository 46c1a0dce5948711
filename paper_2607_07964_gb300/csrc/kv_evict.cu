// kq_kv_evict: the slots of a sequence and head that stay, and the moves that bring them to the front.
//
// Selection: a slot's key is its weight as an order-preserving whole number, above all of them for
// a protected slot. The budget-th largest key is found by four counts over 8 bits each; slots above
// it stay, and of those equal to it the lowest. A kept slot at or beyond the budget moves into a
// free one below it, i-th to i-th, so the two sides never overlap, nothing is copied that already has
// its place, and cutting 64 of 4160 slots moves 64 rows, not 4096.
//
// What bounds it: 8 bytes a slot to read and 2 (D + 8) a move are little (1.3 us and 8 us for 64 heads
// of 20000 slots cut to 4096), so it is the chain of steps: read, four counts, two prefix sums, moves.
// A head's slots are therefore shared by a cluster of up to 8 CTAs, which exchange their counts
// through distributed shared memory; each keeps the keys of its part of the slots in shared memory, a run
// of consecutive slots to a thread, so that ties and the two lists come out in the order of slots by
// prefix sums.
#include <algorithm>
#include <atomic>

#include "kv_common.cuh"

namespace kq {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kCluster = 8;                    // CTAs of a head, at most
constexpr int kKeys = 48 * 1024;               // keys that a CTA holds; beyond them they are made again from memory
constexpr int kMoves = 4;                      // moves of a warp in flight

// Order-preserving key of a slot: protected above every weight, NaN below.
__device__ __forceinline__ uint32_t evict_key(float w, int64_t pos, int64_t from, int64_t sink) {
    if (pos >= from || pos < sink) return 0xFFFFFFFFu;
    if (isnan(w)) return 0u;
    const uint32_t u = __float_as_uint(w == 0.0f ? 0.0f : w);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ uint32_t remote_u32(const void* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(smem_u32(p), rank)) : "memory");
    return v;
}

// Exclusive prefix sum over the block of two 32-bit counts in one word; total receives the sum.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* tmp, uint64_t& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint64_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) tmp[warp] = x;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        if (i < warp) before += tmp[i];
        total += tmp[i];
    }
    return before + x - v;
}

struct Evict {
    KvView c;
    const int32_t *lens, *seen;
    const float* acc;
    const int32_t* pos;
    int64_t S, budget, recent, sink;
    int32_t* lens_out;
    float* acc_out;
    int32_t *pos_out, *lists;
    int* info;
    int32_t per;     // slots of a CTA, a multiple of kThreads
};

__global__ void __launch_bounds__(kThreads) kv_evict_kernel(const Evict e) {
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[256], sum[256], picked[2], counts[3];
    __shared__ uint64_t tmp[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cluster_ctarank();
    uint32_t ctas;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
    const int64_t head = blockIdx.x / ctas;
    const int b = static_cast<int>(head / e.c.kv_heads), h = static_cast<int>(head % e.c.kv_heads);
    const int64_t n = kv_length(e.lens, b, min(kv_capacity(e.c), e.S), e.info);
    const int64_t budget = e.budget;
    if (h == 0 && rank == 0 && tid == 0) e.lens_out[b] = static_cast<int32_t>(min(n, budget));
    const float* acc = e.acc + head * e.S;
    const int32_t* pos = e.pos + head * e.S;
    float* acc_out = e.acc_out + head * e.S;
    int32_t* pos_out = e.pos_out + head * e.S;
    const int64_t first = static_cast<int64_t>(rank) * e.per;
    const int64_t mine = max(static_cast<int64_t>(0), min(static_cast<int64_t>(e.per), n - first));
    const int64_t kept = min(n, budget);
    if (n <= budget) {   // the whole cluster leaves
        for (int64_t j = first + tid; j < first + mine; j += kThreads) {
            if (acc_out != acc) acc_out[j] = acc[j];
            if (pos_out != pos) pos_out[j] = pos[j];
        }
        return;
    }
    const int64_t from = static_cast<int64_t>(e.seen[b]) - e.recent;
    for (int64_t j = tid; j < min(mine, static_cast<int64_t>(kKeys)); j += kThreads)
        keys[j] = evict_key(acc[first + j], pos[first + j], from, e.sink);
    auto key = [&](int64_t j) { return j < kKeys ? keys[j] : evict_key(acc[first + j], pos[first + j], from, e.sink); };

    // ---- the budget-th largest key: 8 bits at a time, from the top
    uint32_t prefix = 0;
    int64_t want = budget;   // how many of the keys that share the prefix stay
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int64_t j0 = 0; j0 < mine; j0 += kThreads) {
            const int64_t j = j0 + tid;
            const uint32_t k = j < mine ? key(j) : 0;
            const bool in = j < mine && (shift == 24 || k >> (shift + 8) == prefix >> (shift + 8));
            // keys of a warp often share their upper bits: one count for all of them
            const uint32_t bin = in ? k >> shift & 255u : 256u, same = __match_any_sync(0xffffffffu, bin);
            if (in && (same & ((1u << lane) - 1)) == 0) atomicAdd(&hist[bin], __popc(same));
        }
        cluster_barrier();
        if (tid < 256) {
            uint32_t s = 0;
            for (uint32_t r = 0; r < ctas; ++r) s += remote_u32(&hist[tid], r);
            sum[tid] = s;
        }
        __syncthreads();
        if (warp == 0) {   // from the largest bin: the one in which the want-th key falls
            uint32_t v[8], s = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i] = sum[255 - (lane * 8 + i)];
            uint32_t x = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            uint32_t before = x - s;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < want && want <= before + static_cast<int64_t>(v[i])) {
                    picked[0] = 255 - (lane * 8 + i);
                    picked[1] = before;
                }
                before += v[i];
            }
        }
        cluster_barrier();   // hist is read by the others until here, picked written
        prefix |= picked[0] << shift;
        want -= picked[1];
    }
    const uint32_t t = prefix;   // want: how many slots equal to it stay, the lowest

    // ---- ties before this CTA, then kept or not, slot by slot: a run of them to a thread
    const int64_t run = (mine + kThreads - 1) / kThreads, j0 = min(tid * run, mine), j1 = min(j0 + run, mine);
    uint32_t eq = 0;
    for (int64_t j = j0; j < j1; ++j) eq += key(j) == t;
    uint64_t total;
    uint64_t ties = block_scan(eq, tmp, total);
    if (tid == 0) counts[0] = static_cast<uint32_t>(total);
    cluster_barrier();
    for (uint32_t r = 0; r < rank; ++r) ties += remote_u32(&counts[0], r);
    uint64_t both = 0;   // holes, and kept slots past the budget in the upper half
    uint64_t tie = ties;
    for (int64_t j = j0; j < j1; ++j) {
        const uint32_t k = key(j);
        const bool keep = k > t || (k == t && static_cast<int64_t>(tie++) < want);
        if (first + j < budget) both += !keep;
        else both += static_cast<uint64_t>(keep) << 32;
    }
    uint64_t at = block_scan(both, tmp, total);
    if (tid == 0) {
        counts[1] = static_cast<uint32_t>(total);
        counts[2] = static_cast<uint32_t>(total >> 32);
    }
    cluster_barrier();
    uint32_t hole_at = static_cast<uint32_t>(at), tail_at = static_cast<uint32_t>(at >> 32), holes = 0;
    for (uint32_t r = 0; r < ctas; ++r) {
        const uint32_t x = remote_u32(&counts[1], r);
        if (r < rank) {
            hole_at += x;
            tail_at += remote_u32(&counts[2], r);
        }
        holes += x;
    }
    int32_t* hole = e.lists + head * 2 * budget;
    int32_t* tail = hole + budget;
    tie = ties;
    for (int64_t j = j0; j < j1; ++j) {
        const uint32_t k = key(j);
        const bool keep = k > t || (k == t && static_cast<int64_t>(tie++) < want);
        if (first + j < budget) {
            if (!keep) hole[hole_at++] = static_cast<int32_t>(first + j);
        } else if (keep) {
            tail[tail_at++] = static_cast<int32_t>(first + j);
        }
    }
    __threadfence();
    cluster_barrier();   // the lists are complete, and no counts are read any more

    // ---- weights and positions of the front, holes left out where the arrays differ; then the moves
    for (int64_t j = first + tid; j < min(first + mine, kept); j += kThreads) {
        if (acc_out != acc) acc_out[j] = acc[j];
        if (pos_out != pos) pos_out[j] = pos[j];
    }
    cluster_barrier();
    const int words = e.c.dim / 8;   // of a row of codes
    for (int64_t m0 = static_cast<int64_t>(warp * ctas + rank) * kMoves; m0 < holes; m0 += static_cast<int64_t>(kWarps) * ctas * kMoves) {
        uint8_t* dst[kMoves];
        uint32_t code[kMoves], prm[kMoves], extra[kMoves];
        int32_t to[kMoves], td[kMoves];
#pragma unroll
        for (int i = 0; i < kMoves; ++i) {
            dst[i] = nullptr;
            if (m0 + i >= holes) continue;
            to[i] = hole[m0 + i];
            const int32_t src_slot = tail[m0 + i];
            const uint8_t* src = kv_granule(e.c, b, h, src_slot);
            dst[i] = kv_granule(e.c, b, h, to[i]);
            if (!src || !dst[i]) {
                record_error(e.info, -KQ_ERR_INVALID_ARG);
                dst[i] = nullptr;
                continue;
            }
            const int ts = src_slot % kGranule;
            td[i] = to[i] % kGranule;
            // lanes 0 .. words - 1 the key's codes, the next as many the value's
            if (lane < 2 * words)
                code[i] = reinterpret_cast<const uint32_t*>(src + kv_code_at(e.c.dim, lane >= words, ts))[lane % words];
            if (lane < 2) {
                prm[i] = *reinterpret_cast<const uint32_t*>(src + kv_param_at(e.c.dim, lane, ts));
                extra[i] = lane ? static_cast<uint32_t>(pos[src_slot]) : __float_as_uint(acc[src_slot]);
            }
        }
#pragma unroll
        for (int i = 0; i < kMoves; ++i) {
            if (!dst[i]) continue;
            if (lane < 2 * words)
                reinterpret_cast<uint32_t*>(dst[i] + kv_code_at(e.c.dim, lane >= words, td[i]))[lane % words] = code[i];
            if (lane < 2) {
                *reinterpret_cast<uint32_t*>(dst[i] + kv_param_at(e.c.dim, lane, td[i])) = prm[i];
                if (lane) pos_out[to[i]] = static_cast<int32_t>(extra[i]);
                else acc_out[to[i]] = __uint_as_float(extra[i]);
            }
        }
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
    static std::atomic<uint64_t> done{0};
    KQ_TRY(once_per_device(done, [] {
        KQ_CUDA(cudaFuncSetAttribute(kv_evict_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(kKeys * sizeof(uint32_t))));
        return KQ_OK;
    }));
    // CTAs of a head: one up to 4096 slots, where the exchanges between CTAs would cost more than
    // they save, or where the heads fill the GPU; else as many as keep 2048 slots each, up to a cluster.
    const int64_t most = std::min(S, kv_capacity(c));
    int ctas = 1;
    while (ctas < kCluster && most > 4096 && most > 2048 * ctas && c.batch * c.kv_heads * ctas < 2 * num_sms()) ctas *= 2;
    const Evict e = {c, lens, seen, acc, pos, S, budget, recent, sink, lens_out, acc_out, pos_out, static_cast<int32_t*>(ws), info,
                     static_cast<int32_t>(cdiv(cdiv(most, ctas), kThreads) * kThreads)};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(c.batch * c.kv_heads * ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = std::min<size_t>(kKeys, e.per) * sizeof(uint32_t);
    cfg.stream = reinterpret_cast<cudaStream_t>(stream_);
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {static_cast<unsigned>(ctas), 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = 1;
    KQ_CUDA(cudaLaunchKernelEx(&cfg, kv_evict_kernel, e));
    KQ_LAUNCH_CHECK("kv_evict_kernel");
    return KQ_OK;
}
