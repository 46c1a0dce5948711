// kq_kv_evict: the slots of a sequence and head that stay, and the moves that bring them to the front.
//
// Selection: a slot's key is its weight as an order-preserving whole number, above all of them for
// a protected slot. The budget-th largest key is found by up to four counts over 8 bits each; slots
// above it stay, and of those equal to it the lowest. A kept slot at or beyond the budget moves into a
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
constexpr int kMoves = 16;                     // moves of a warp in flight

// Order-preserving key of a slot: protected above every weight, NaN below.
__device__ __forceinline__ uint32_t evict_key(float w, int32_t pos, int32_t from, int32_t sink) {
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
    int64_t S;
    int32_t budget, recent, sink;
    int32_t* lens_out;
    float* acc_out;
    int32_t *pos_out, *lists;
    int* info;
    int32_t ctas, per;   // CTAs of a head, slots of each: a multiple of kThreads
};

// ONE: a head has one CTA, and nothing to exchange. FITS: a CTA's keys fit its shared memory.
template <bool ONE, bool FITS>
__global__ void __launch_bounds__(kThreads) kv_evict_kernel(const Evict e) {
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[4][256], sum[256], picked[3], counts[6];   // a count for each digit: none is cleared while read
    __shared__ uint64_t tmp[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = ONE ? 0 : static_cast<int>(cluster_ctarank()), ctas = ONE ? 1 : e.ctas;
    auto sync = [] {
        if constexpr (ONE) __syncthreads();
        else cluster_barrier();
    };
    auto count_of = [&](int i, int r) { return ONE ? counts[i] : remote_u32(&counts[i], r); };
    const int head = blockIdx.x / ctas;
    const int b = head / e.c.kv_heads, h = head % e.c.kv_heads;
    const int n = static_cast<int>(kv_length(e.lens, b, min(kv_capacity(e.c), e.S), e.info));
    const int budget = e.budget;
    if (h == 0 && rank == 0 && tid == 0) e.lens_out[b] = min(n, budget);
    const float* acc = e.acc + head * e.S;
    const int32_t* pos = e.pos + head * e.S;
    float* acc_out = e.acc_out + head * e.S;
    int32_t* pos_out = e.pos_out + head * e.S;
    const int first = rank * e.per, mine = max(0, min(e.per, n - first));   // first < 2^31: no further than S and a part
    // the front's weights and positions, free slots among them, where the arrays differ
    auto copy = [&](int j, float w, int32_t q) {
        if (first + j >= budget) return;
        if (acc_out != acc) acc_out[first + j] = w;
        if (pos_out != pos) pos_out[first + j] = q;
    };
    if (n <= budget) {   // the whole cluster leaves
        for (int j = tid; j < mine; j += kThreads) copy(j, acc[first + j], pos[first + j]);
        return;
    }
    const int from = static_cast<int>(max(static_cast<int64_t>(INT32_MIN), static_cast<int64_t>(e.seen[b]) - e.recent));
    auto made = [&](int j) { return evict_key(acc[first + j], pos[first + j], from, e.sink); };
    for (int i = tid; i < 4 * 256; i += kThreads) hist[0][i] = 0;
    if (tid == 0) counts[3] = 0xFFFFFFFFu, counts[4] = counts[5] = 0;
    __syncthreads();
    uint32_t low = 0xFFFFFFFFu, high = 0, safe = 0;   // of the keys that are not protected; how many are
    auto note = [&](uint32_t k) {
        safe += k == 0xFFFFFFFFu;
        low = min(low, k);
        if (k != 0xFFFFFFFFu) high = max(high, k);
    };
    {
        const int held = FITS ? mine : min(mine, kKeys);
        int j = tid;
        for (; j + 3 * kThreads < held; j += 4 * kThreads) {
            float w[4];
            int32_t q[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = acc[first + j + i * kThreads], q[i] = pos[first + j + i * kThreads];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t k = evict_key(w[i], q[i], from, e.sink);
                keys[j + i * kThreads] = k;
                copy(j + i * kThreads, w[i], q[i]);
                note(k);
            }
        }
        for (; j < mine; j += kThreads) {
            const float w = acc[first + j];
            const int32_t q = pos[first + j];
            const uint32_t k = evict_key(w, q, from, e.sink);
            if (FITS || j < kKeys) keys[j] = k;
            copy(j, w, q);
            note(k);
        }
    }
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    safe = __reduce_add_sync(0xffffffffu, safe);
    if (lane == 0) {
        atomicMin(&counts[3], low);
        atomicMax(&counts[4], high);
        atomicAdd(&counts[5], safe);
    }
    sync();
    low = 0xFFFFFFFFu, high = 0, safe = 0;
    for (int r = 0; r < ctas; ++r) {
        low = min(low, count_of(3, r));
        high = max(high, count_of(4, r));
        safe += count_of(5, r);
    }
    auto key = [&](int j) { return FITS || j < kKeys ? keys[j] : made(j); };

    // ---- the budget-th largest key: among the others once the protected slots have their places, by their distance
    // from the smallest, 8 bits at a time from the first that any has (weights share a few exponents; their
    // distances spread over the bins)
    const bool crowd = safe >= static_cast<uint32_t>(budget);   // the protected alone fill the budget, the lowest first
    uint32_t prefix = 0, want = crowd ? budget : budget - safe;   // want: how many of the keys that share the prefix stay
    const int bits = crowd ? 0 : 32 - __clz(high - low);
    for (int digit = 0, shift = bits - 8; shift > -8; ++digit, shift -= 8) {
        uint32_t* const bins = hist[digit];
        const int down = max(shift, 0), above = shift + 8;   // the last digit may have fewer than 8 bits
        for (int j = tid; j < mine; j += kThreads) {
            const uint32_t k = key(j) - low;
            if (k > high - low) continue;   // protected
            if (above < 32 && (k ^ prefix) >> above) continue;
            atomicAdd(&bins[(k & (above < 32 ? (1u << above) - 1 : 0xFFFFFFFFu)) >> down], 1u);
        }
        sync();
        if constexpr (!ONE) {
            if (tid < 256) {
                uint32_t s = 0;
#pragma unroll
                for (int r = 0; r < kCluster; ++r)
                    if (r < ctas) s += remote_u32(&bins[tid], r);
                sum[tid] = s;
            }
            __syncthreads();
        }
        if (warp == 0) {   // from the largest bin: the one in which the want-th key falls
            uint32_t v[8], s = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i] = (ONE ? bins : sum)[255 - (lane * 8 + i)];
            uint32_t x = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            uint32_t before = x - s;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < want && want <= before + v[i]) {
                    picked[0] = 255 - (lane * 8 + i);
                    picked[1] = before;
                    picked[2] = v[i];
                }
                before += v[i];
            }
        }
        __syncthreads();   // picked by each CTA for itself
        prefix |= picked[0] << down;
        want -= picked[1];
    }
    // slots equal to the threshold: all of them stay, unless the last bin held more than that
    const bool tied = bits <= 0 || picked[2] != want;
    const uint32_t t = crowd ? 0xFFFFFFFFu : low + prefix;   // want: how many slots equal to it stay, the lowest

    // ---- ties before this CTA, then kept or not, slot by slot: a run of them to a thread
    const int run = (mine + kThreads - 1) / kThreads | 1;   // odd: neighbouring threads in different banks
    const int j0 = min(tid * run, mine), j1 = min(j0 + run, mine);
    uint64_t total;
    uint32_t ties = 0;
    if (tied) {
        uint32_t eq = 0;
        for (int j = j0; j < j1; ++j) eq += key(j) == t;
        ties = static_cast<uint32_t>(block_scan(eq, tmp, total));
        if constexpr (!ONE) {
            if (tid == 0) counts[0] = static_cast<uint32_t>(total);
            sync();
            for (int r = 0; r < rank; ++r) ties += count_of(0, r);
        }
    } else {
        want = 0xFFFFFFFFu;
    }
    uint32_t holes_here = 0, tails_here = 0, tie = ties;
    const int edge = budget - first;   // this CTA's slots below the budget
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = key(j);
        const bool keep = k > t || (k == t && tie++ < want);
        holes_here += j < edge && !keep;
        tails_here += j >= edge && keep;
    }
    const uint64_t at = block_scan(holes_here | static_cast<uint64_t>(tails_here) << 32, tmp, total);
    uint32_t hole_at = static_cast<uint32_t>(at), tail_at = static_cast<uint32_t>(at >> 32), holes = static_cast<uint32_t>(total);
    if constexpr (!ONE) {
        if (tid == 0) {
            counts[1] = static_cast<uint32_t>(total);
            counts[2] = static_cast<uint32_t>(total >> 32);
        }
        sync();
        holes = 0;
        for (int r = 0; r < ctas; ++r) {
            const uint32_t x = count_of(1, r);
            if (r < rank) {
                hole_at += x;
                tail_at += count_of(2, r);
            }
            holes += x;
        }
    }
    int32_t* hole = e.lists + static_cast<int64_t>(head) * 2 * budget;
    int32_t* tail = hole + budget;
    tie = ties;
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = key(j);
        const bool keep = k > t || (k == t && tie++ < want);
        if (j < edge && !keep && KQ_IN_RANGE(hole_at, budget)) hole[hole_at++] = first + j;
        if (j >= edge && keep && KQ_IN_RANGE(tail_at, budget)) tail[tail_at++] = first + j;
    }
    sync();   // the lists and the fronts are complete, and no counts are read any more

    // ---- the moves: a lane finds both places of one and takes its parameters, weight and position; then the warp
    // copies the code rows of one after the other
    const int words = e.c.dim / 8, row = e.c.dim / 2;   // words and bytes of a row of codes
    // lanes 0 .. words - 1 the key's codes, the next as many the value's
    const int in_row = (lane >= words ? kGranule * row + (lane - words) * 4 : lane * 4);
    const bool copies = lane < 2 * words;
    const uint32_t chunk = min(32u, max(4u, (holes + kWarps * ctas - 1) / (kWarps * ctas)));
    for (uint32_t m0 = (warp * ctas + rank) * chunk; m0 < holes; m0 += kWarps * ctas * chunk) {
        const uint32_t here = min(chunk, holes - m0);
        const uint8_t* src = nullptr;
        uint8_t* dst = nullptr;
        if (lane < here) {
            const int to = hole[m0 + lane], at = tail[m0 + lane];
            src = kv_granule(e.c, b, h, at);
            dst = kv_granule(e.c, b, h, to);
            if (src && dst) {
                const int ts = at % kGranule, td = to % kGranule;
                const float w = acc[at];
                const int32_t q = pos[at];
                uint32_t prm[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) prm[i] = *reinterpret_cast<const uint32_t*>(src + kv_param_at(e.c.dim, i, ts));
#pragma unroll
                for (int i = 0; i < 2; ++i) *reinterpret_cast<uint32_t*>(dst + kv_param_at(e.c.dim, i, td)) = prm[i];
                if (KQ_IN_RANGE(to, e.S)) {
                    acc_out[to] = w;
                    pos_out[to] = q;
                }
                src += ts * row;
                dst += td * row;
            } else {
                record_error(e.info, -KQ_ERR_INVALID_ARG);
                dst = nullptr;
            }
        }
        for (uint32_t k0 = 0; k0 < here; k0 += kMoves) {
            uint32_t code[kMoves];
#pragma unroll
            for (int i = 0; i < kMoves; ++i) {
                const uint64_t s = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(src), k0 + i & 31);
                const uint64_t d = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(dst), k0 + i & 31);
                if (k0 + i < here && d && copies) code[i] = *reinterpret_cast<const uint32_t*>(s + in_row);
            }
#pragma unroll
            for (int i = 0; i < kMoves; ++i) {
                const uint64_t d = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(dst), k0 + i & 31);
                if (k0 + i < here && d && copies && KQ_IN_RANGE(d + in_row - reinterpret_cast<uint64_t>(e.c.data), kv_pool_bytes(e.c) - 3))
                    *reinterpret_cast<uint32_t*>(d + in_row) = code[i];
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
    if (!lens || !acc || !pos || !seen || !lens_out || !acc_out || !pos_out || S < 1 ||
        kv_overlap(lens_out, c.batch, lens, c.batch) || kv_overlap(lens_out, c.batch, seen, c.batch) ||   // other blocks read them
        S > 0x7fffffffll - (1 << 20) || budget < 1 || recent < 0 || sink < 0 || recent > budget || sink > budget - recent) {
        set_error("kq_kv_evict: arrays must not be NULL, lens_out apart from lens and seen, budget >= 1, recent + sink <= budget");
        return KQ_ERR_INVALID_ARG;
    }
    budget = std::min(budget, S);
    recent = std::min<int64_t>(recent, 0x7fffffff);
    sink = std::min<int64_t>(sink, 0x7fffffff);
    const size_t need = kq_kv_evict_workspace(c.batch, c.kv_heads, S, budget);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("kq_kv_evict: workspace must be 256-byte aligned and hold %zu bytes", need);
        return KQ_ERR_WORKSPACE;
    }
    static std::atomic<uint64_t> done{0};
    KQ_TRY(once_per_device(done, [] {
        const int most_smem = static_cast<int>(kKeys * sizeof(uint32_t));
        KQ_CUDA(cudaFuncSetAttribute(kv_evict_kernel<true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem));
        KQ_CUDA(cudaFuncSetAttribute(kv_evict_kernel<true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem));
        KQ_CUDA(cudaFuncSetAttribute(kv_evict_kernel<false, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem));
        KQ_CUDA(cudaFuncSetAttribute(kv_evict_kernel<false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most_smem));
        return KQ_OK;
    }));
    // CTAs of a head: one up to 4096 slots, where the exchanges between CTAs would cost more than
    // they save, or where the heads fill the GPU; else as many as keep 2048 slots each, up to a cluster.
    const int64_t most = std::min(S, kv_capacity(c));
    int ctas = 1;
    while (ctas < kCluster && most > 4096 && most > 2048 * ctas && c.batch * c.kv_heads * ctas <= num_sms()) ctas *= 2;
    const Evict e = {c, lens, seen, acc, pos, S, static_cast<int32_t>(budget), static_cast<int32_t>(recent), static_cast<int32_t>(sink),
                     lens_out, acc_out, pos_out, static_cast<int32_t*>(ws), info, ctas,
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
    const bool fits = e.per <= kKeys;
    KQ_CUDA(ctas == 1 ? (fits ? cudaLaunchKernelEx(&cfg, kv_evict_kernel<true, true>, e) : cudaLaunchKernelEx(&cfg, kv_evict_kernel<true, false>, e))
                      : (fits ? cudaLaunchKernelEx(&cfg, kv_evict_kernel<false, true>, e) : cudaLaunchKernelEx(&cfg, kv_evict_kernel<false, false>, e)));
    KQ_LAUNCH_CHECK("kv_evict_kernel");
    return KQ_OK;
}
