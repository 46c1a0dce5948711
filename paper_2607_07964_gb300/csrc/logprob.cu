// kq_token_logprobs and kq_token_logprobs_grad: rows of logits, each read once.
//
// Mathematics. With t_v = log2(e) x_v - r for a reference r (in powers of two) near the maximum,
//     Z = sum 2^t,  lse = (r + log2 Z) ln 2,  logp_v = (t_v - log2 Z) ln 2,
//     entropy = (log2 Z - sum 2^t t / Z) ln 2.
// A thread keeps a reference of its own, moved only when a value passes it by 2^kSlack, so Z and
// sum 2^t t need no rescaling in the common step; r differs from the maximum by so little that the
// entropy's two terms do not cancel beyond a few units. t is formed by one fma, the same for every
// use, so a rounding of r (kHuge bounds it) cancels from logp and entropy.
//
// The largest `top` values: a bound that at least `top` of the threads' maxima reach, and the row's groups
// of kAhead (kWideAhead) vectors whose own maximum, noted in 16 bits in shared memory along the way, reaches it
// too: only those few are read again. (Going through all values of the threads that reach the bound
// instead reads a third of the row a second time, when it has left L2.)
//
// What bounds it: with V = 128000 in bf16 a row is 256 KB, 5.7 us of an SM's share of the memory
// bandwidth, against about 6 instructions a value (3 us) and 1.5 us for the joint steps, which
// other rows' blocks on the SM cover. The gradient reads and writes a row once.
#include <algorithm>
#include <atomic>

#include "kv_common.cuh"

namespace kq {
namespace {

constexpr int kThreads = 256;             // of a block where there are rows for every SM, and of the gradient's
constexpr int kNarrow = 64, kMedium = 128; // of one for a row of less than kShortRow, kMiddleRow bytes
constexpr int kShortRow = 12288, kMiddleRow = 98304;
constexpr int kWide = 1024;               // where there are few rows
constexpr int kSplit = 512;               // where there are two to an SM, or so few that a cluster takes a row
constexpr int kCluster = 8, kSplitBytes = 32768;   // of that many blocks at most, with no less than that of the row each
constexpr int kAhead = 4;                 // 16-byte loads of a thread in flight
constexpr int kWideAhead = 8;             // of one in a block that has the SM to itself
constexpr int kList = 1024;               // candidates for the top values
constexpr int kGroups = 256;              // groups that are looked through for them
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kSlack = 4.0f;
constexpr float kFloor = -2.0e38f;        // what a masked logit counts as: 2^t = 0 and t a number
// Rows whose maximum is beyond this, or -infinity, go the careful way. The reference's rounding, in every t alike, is
// at most 2^6 here, so that neither 2^t nor Z leaves the range and the terms that cancel stay below 2^7; and log2(e)
// kFloor less a reference is a number, whose share 0 t is 0. (2^30 leaves rows shifted by -1e9 to the fast way.)
constexpr float kHuge = 0x1p30f;

__device__ __forceinline__ float value(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float value(const __nv_bfloat16* p, int64_t i) { return __bfloat162float(p[i]); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Larger for a larger logit, then for a smaller index; NaN above every number; never 0.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t i) {
    uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    u = isnan(x) ? 0xFFFFFFFFu : (u >> 31) ? ~u : (u | 0x80000000u);
    return (static_cast<uint64_t>(u) << 32) | (0xFFFFFFFFu - i);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xFFFFFFFFu - static_cast<uint32_t>(k); }
__device__ __forceinline__ float key_value(uint64_t k) {
    const uint32_t u = static_cast<uint32_t>(k >> 32);
    return __uint_as_float((u >> 31) ? u & 0x7FFFFFFFu : ~u);
}

// The values of a 16-byte vector, no lower than kFloor (a NaN stays one), and their true maximum
// (NaN left out).
template <typename T>
__device__ __forceinline__ float unpack(const uint4& u, float (&x)[16 / sizeof(T)]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if constexpr (sizeof(T) == 2) {
        constexpr uint32_t floor2 = 0xFF16FF16u;   // bf16(kFloor) twice
        uint32_t a, b, m;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(w[0]), "r"(w[1]));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(w[2]), "r"(w[3]));
        asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t c;
            asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(w[i]), "r"(floor2));
            x[2 * i] = __uint_as_float(c << 16);
            x[2 * i + 1] = __uint_as_float(c & 0xFFFF0000u);
        }
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(x[i]) : "f"(__uint_as_float(w[i])), "f"(kFloor));
        return fmaxf(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])), fmaxf(__uint_as_float(w[2]), __uint_as_float(w[3])));
    }
}

template <int NT, typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* tmp, F f) {
    for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = v;
    __syncthreads();
    v = tmp[threadIdx.x % (NT / 32)];
    for (int o = NT / 64; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float sum2(float a, float b) { return a + b; }

__device__ __forceinline__ uint32_t remote_u32(const void* p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_shared(smem_u32(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ float remote_f32(const float* p, uint32_t rank) { return __uint_as_float(remote_u32(p, rank)); }

// ln p of a logit; one masked with its type's lowest number would overflow in powers of two.
__device__ __forceinline__ float logp_of(float x, float r2, float lz2) {
    return x < kFloor ? x - (r2 + lz2) * kLn2 : fminf(0.0f, (fmaf(x, kLog2e, -r2) - lz2) * kLn2);
}

struct Out {
    float *logp, *entropy, *lse;
    int32_t* top_id;
    float* top_logp;
    int* info;
};

// A row with a NaN or an infinite maximum, or whose values leave the range of the fast way: one value
// at a time, the top values one after the other.
template <typename T, int NT>
__device__ __noinline__ void careful_row(const T* x, int64_t r, int64_t V, int64_t y, int top, const Out& out, uint64_t* tmp64) {
    float* tmp = reinterpret_cast<float*>(tmp64);
    float m = -INFINITY;
    int bad = 0;
    for (int64_t i = threadIdx.x; i < V; i += NT) {
        const float v = value(x, i);
        bad |= isnan(v) || v == INFINITY;
        m = fmaxf(m, v);
    }
    m = block_reduce<NT>(m, tmp, [](float a, float b) { return fmaxf(a, b); });
    bad = __syncthreads_or(bad);
    float z = 0.0f, w = 0.0f;
    for (int64_t i = threadIdx.x; i < V; i += NT) {
        const float d = value(x, i) - m;
        if (d > -INFINITY) {
            const float e = expf(d);
            z += e;
            if (e > 0.0f) w -= e * d;
        }
    }
    z = block_reduce<NT>(z, tmp, [](float a, float b) { return a + b; });
    w = block_reduce<NT>(w, tmp, [](float a, float b) { return a + b; });
    const float lz = logf(z);
    const bool none = m == -INFINITY;
    if (threadIdx.x == 0) {
        out.logp[r] = y < 0 ? 0.0f : y >= V || bad ? NAN : none ? -INFINITY : value(x, y) - m - lz;
        if (out.entropy) out.entropy[r] = bad ? NAN : none ? 0.0f : lz + w / z;
        if (out.lse) out.lse[r] = bad ? NAN : none ? -INFINITY : m + lz;
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t best = 0;
        for (int64_t i = threadIdx.x; i < V; i += NT) {
            const uint64_t key = rank_key(value(x, i), static_cast<uint32_t>(i));
            if (key < last && key > best) best = key;
        }
        best = block_reduce<NT>(best, tmp64, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        last = best;
        if (threadIdx.x == 0) {
            out.top_id[r * top + k] = static_cast<int32_t>(key_index(best));
            out.top_logp[r * top + k] = bad ? NAN : none ? -INFINITY : key_value(best) - m - lz;
        }
    }
}

// Value e of a 16-byte vector.
template <typename T>
__device__ __forceinline__ float value_of(const uint4& u, int e) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    return __uint_as_float(sizeof(T) == 4 ? w[e % 4] : e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
}
// Candidates for the top values: those from the bound up, by value and index.
struct Offers {
    uint64_t bound;
    uint64_t* list;
    int* n;

    __device__ __forceinline__ void add(uint64_t k) const {
        if (k < bound) return;
        const int at = atomicAdd(n, 1);
        if (at < kList) list[at] = k;
    }
    template <typename T>
    __device__ __forceinline__ void add_vector(const uint4* v, uint32_t first) const {
        const uint4 u = __ldg(v);
#pragma unroll
        for (int e = 0; e < static_cast<int>(16 / sizeof(T)); ++e) add(rank_key(value_of<T>(u, e), first + e));
    }
};
// A thread's share of a row: vectors threadIdx.x, threadIdx.x + NT, .. of nvec, A of them a group.
struct Mine {
    const uint4* xv;
    int nvec, groups, best_group;   // the group with the largest value
    uint32_t first;                 // index in the row of the first vector's first value
    uint32_t most;                  // order of the largest value
    uint64_t edge;                  // key of the thread's value outside the vectors, or 0
};
// Too many near the bound's value: the bound becomes the top-th largest of the threads' first largest values by value and
// index (complements, the largest first; an index is below 2^20), and the groups that may hold something from there up are
// read, on a list by all threads, or else each by its own: any number of float32 groups can share the bound's upper half
// (4096 rows of 32000 fp32 logits, 20 top values: 105 us; all near 100 within 0.03, 126 us; all equal, 130 us).
template <typename T, int NT, int A>
__device__ __forceinline__ void second_look(const Mine& a, const uint16_t* group_max, int top, uint64_t* list, int* n_list,
                                            int* groups, int* n_groups) {
    constexpr int E = 16 / sizeof(T);
    uint64_t key = a.edge, bound = 0;
    const int at0 = a.best_group * A * NT + static_cast<int>(threadIdx.x);
    uint4 u[A];
#pragma unroll
    for (int i = 0; i < A; ++i)
        if (at0 + i * NT < a.nvec) u[i] = __ldg(a.xv + at0 + i * NT);
#pragma unroll
    for (int i = 0; i < A; ++i) {
        if (at0 + i * NT >= a.nvec) break;
#pragma unroll
        for (int e = 0; e < E; ++e)
            key = max(key, rank_key(value_of<T>(u[i], e), a.first + static_cast<uint32_t>((at0 + i * NT) * E + e)));
    }
    for (int bit = 63; bit >= 0; --bit) {
        if (bit < 32 && bit >= 20) {
            bound |= 1ull << bit;
            continue;
        }
        const uint64_t cand = bound | (1ull << bit);
        if (__syncthreads_count(key >= cand) >= top) bound = cand;
    }
    if (threadIdx.x == 0) *n_list = *n_groups = 0;
    __syncthreads();
    const Offers offers = {bound, list, n_list};
    if (a.edge) offers.add(a.edge);
    const uint32_t bound_value = static_cast<uint32_t>(bound >> 32), bound_index = key_index(bound);
    // Where no value of a group is above the bound's (in bf16 the upper half says so, in float32 the thread's largest
    // can), one that begins behind the bound's index has nothing to offer.
    auto each_group = [&](auto f) {
        for (int g = 0; g < a.groups && a.most >= bound_value; ++g) {
            const uint32_t gm = group_max[g * NT + threadIdx.x];
            const int first = g * A * NT + static_cast<int>(threadIdx.x);
            const bool equal = sizeof(T) == 2 ? gm == bound_value >> 16 : a.most == bound_value;
            if (gm < bound_value >> 16 || (equal && a.first + static_cast<uint32_t>(first * E) > bound_index)) continue;
            f(first);
        }
    };
    auto read = [&](int at) {
        if (at < a.nvec) offers.add_vector<T>(a.xv + at, a.first + static_cast<uint32_t>(at * E));
    };
    each_group([&](int first) {
        const int at = atomicAdd(n_groups, 1);
        if (at < kGroups) groups[at] = first;
    });
    __syncthreads();
    if (*n_groups <= kGroups) {
        for (int q = threadIdx.x; q < *n_groups * A; q += NT) read(groups[q / A] + q % A * NT);
    } else {
        each_group([&](int first) {
            for (int i = 0; i < A; ++i) read(first + i * NT);
        });
    }
    __syncthreads();
}

// SPLIT: a cluster takes a row, each block an equal run of `part` values of it.
template <typename T, int NT, bool SPLIT>
__global__ void __launch_bounds__(NT, NT >= kSplit ? 1 : 1536 / NT) logprob_kernel(const T* __restrict__ logits, int64_t row_len,
                                                                                   int64_t ld, const int64_t* __restrict__ target,
                                                                                   int top, Out out, int parts, int part) {
    constexpr int E = 16 / sizeof(T), kWarps = NT / 32, A = NT == kWide ? kWideAhead : kAhead;
    __shared__ uint64_t tmp64[kWarps], list[kList], mine_top[KQ_LOGPROBS_MAX_TOP];
    __shared__ __align__(16) float tmp[2][kWarps][4];
    __shared__ float stat[4];   // this block's maximum, reference and sums, and
    __shared__ int failed;      // whether its top values went past its lists: read by the row's other blocks
    __shared__ int groups[kGroups], n_groups, n_list;
    extern __shared__ uint16_t group_max[];   // [group of a thread][thread]: upper half of the maximum's order
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = SPLIT ? static_cast<int>(cluster_ctarank()) : 0;
    const int64_t r = SPLIT ? blockIdx.x / parts : blockIdx.x;
    const int64_t y = target[r];
    const uint32_t base = SPLIT ? static_cast<uint32_t>(rank) * part : 0;   // this block's first value in the row
    const T* const row = logits + r * ld;
    const T* x = row + base;
    const int64_t V = SPLIT ? max(static_cast<int64_t>(0), min(static_cast<int64_t>(part), row_len - base)) : row_len;
    // vectors of 16 bytes between the first and the last aligned address, and the few values around them
    const int head = static_cast<int>(min(V, static_cast<int64_t>((16 - (reinterpret_cast<uintptr_t>(x) & 15)) % 16 / sizeof(T))));
    const uint4* xv = reinterpret_cast<const uint4*>(x + head);
    const int nvec = static_cast<int>((V - head) / E);
    const int tail = static_cast<int>(V - head) - nvec * E, edge = head + tail;
    const int my_edge = tid < edge ? (tid < head ? tid : head + nvec * E + tid - head) : -1;

    float ref = kFloor, ref2 = 0.0f, z = 0.0f, w = 0.0f, best = -INFINITY;
    int best_group = 0, n_mine = 0;   // of this thread's groups
    auto take = [&](float top_value, const float* v, int n) {
        if (top_value > ref + kSlack) {
            // the rounded product, in the difference as in t: not to be fused with the subtraction
            const float nr2 = __fmul_rn(top_value, kLog2e), f = ref == kFloor ? 0.0f : ex2(ref2 - nr2);
            w = f > 0.0f ? f * fmaf(z, ref2 - nr2, w) : 0.0f;
            z *= f;
            ref = top_value;
            ref2 = nr2;
        }
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float t = fmaf(v[i], kLog2e, -ref2), e = ex2(t);
            z += e;
            w = fmaf(e, t, w);
        }
    };
    // the values' order as whole numbers, and its upper half: all of a bf16 value's
    auto order = [](float v) { return static_cast<uint32_t>(rank_key(v, 0) >> 32); };
    int j = tid;
    for (; j + (A - 1) * NT < nvec; j += A * NT) {
        uint4 u[A];
#pragma unroll
        for (int i = 0; i < A; ++i) u[i] = __ldg(xv + j + i * NT);
        float gm = -INFINITY;
#pragma unroll
        for (int i = 0; i < A; ++i) {
            float v[E];
            const float m = unpack<T>(u[i], v);
            gm = fmaxf(gm, m);
            take(m, v, E);
        }
        if (gm > best) {
            best = gm;
            best_group = n_mine;
        }
        if (top) group_max[n_mine * NT + tid] = static_cast<uint16_t>(order(gm) >> 16);
        ++n_mine;
    }
    if (j < nvec) {
        uint4 u[A - 1];
#pragma unroll
        for (int i = 0; i < A - 1; ++i)
            if (j + i * NT < nvec) u[i] = __ldg(xv + j + i * NT);
        float gm = -INFINITY;
#pragma unroll
        for (int i = 0; i < A - 1; ++i) {
            if (j + i * NT >= nvec) break;
            float v[E];
            const float m = unpack<T>(u[i], v);
            gm = fmaxf(gm, m);
            take(m, v, E);
        }
        if (gm > best) {
            best = gm;
            best_group = n_mine;
        }
        if (top) group_max[n_mine * NT + tid] = static_cast<uint16_t>(order(gm) >> 16);
        ++n_mine;
    }
    float ev = -INFINITY;
    if (my_edge >= 0) {
        ev = value(x, my_edge);
        float c[1];
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(c[0]) : "f"(ev), "f"(kFloor));
        take(ev, c, 1);
    }
    // ---- the sums about one reference
    const bool has = tid < nvec || my_edge >= 0;
    const float mine = fmaxf(best, ev);
    float m = mine, low = has ? mine : INFINITY, r2 = ref == kFloor ? kFloor : ref2;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
        r2 = fmaxf(r2, __shfl_xor_sync(0xffffffffu, r2, o));
    }
    if (lane == 0) tmp[0][warp][0] = m, tmp[0][warp][1] = low, tmp[0][warp][2] = r2;
    __syncthreads();
    {
        const float4 q = *reinterpret_cast<const float4*>(tmp[0][lane % kWarps]);
        m = q.x, low = q.y, r2 = q.z;
    }
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
        r2 = fmaxf(r2, __shfl_xor_sync(0xffffffffu, r2, o));
    }
    {
        const float f = ref == kFloor ? 0.0f : ex2(ref2 - r2);
        w = f > 0.0f ? f * fmaf(z, ref2 - r2, w) : 0.0f;
        z *= f;   // a NaN stays one
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        z += __shfl_xor_sync(0xffffffffu, z, o);
        w += __shfl_xor_sync(0xffffffffu, w, o);
    }
    if (lane == 0) tmp[1][warp][0] = z, tmp[1][warp][1] = w;
    __syncthreads();
    z = tmp[1][lane % kWarps][0], w = tmp[1][lane % kWarps][1];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) {
        z += __shfl_xor_sync(0xffffffffu, z, o);
        w += __shfl_xor_sync(0xffffffffu, w, o);
    }
    float row_max = m;
    if constexpr (SPLIT) {   // the row's, from its blocks' in order
        if (tid == 0) {
            stat[0] = m, stat[1] = r2, stat[2] = z, stat[3] = w;
            failed = 0;
        }
        if (tid < KQ_LOGPROBS_MAX_TOP) mine_top[tid] = 0;
        cluster_barrier();
        float all_r2 = kFloor;
        for (int i = 0; i < parts; ++i) {
            row_max = fmaxf(row_max, remote_f32(&stat[0], i));
            all_r2 = fmaxf(all_r2, remote_f32(&stat[1], i));
        }
        z = w = 0.0f;
        for (int i = 0; i < parts; ++i) {
            const float ri = remote_f32(&stat[1], i), zi = remote_f32(&stat[2], i), wi = remote_f32(&stat[3], i);
            const float f = ri == kFloor ? 0.0f : ex2(ri - all_r2);
            z += zi * f;   // a NaN stays one
            if (f > 0.0f) w += f * fmaf(zi, ri - all_r2, wi);
        }
        r2 = all_r2;
    }
    if (y >= row_len && tid == 0 && rank == 0) record_error(out.info, -KQ_ERR_INVALID_ARG);
    if (!(row_max > -kHuge && row_max < kHuge && z < INFINITY)) {   // false for a NaN in z
        if constexpr (SPLIT) cluster_barrier();   // no block leaves while another reads its part of the row's sums
        if (rank == 0) careful_row<T, NT>(row, r, row_len, y, top, out, tmp64);
        return;
    }
    const float lz2 = log2f(z);
    if (tid == 0 && rank == 0) {
        out.logp[r] = y < 0 ? 0.0f : y >= row_len ? NAN : logp_of(value(row, y), r2, lz2);
        if (out.entropy) out.entropy[r] = fmaxf(0.0f, (lz2 - w / z) * kLn2);
        if (out.lse) out.lse[r] = (r2 + lz2) * kLn2;
    }
    if (top == 0) {
        if constexpr (SPLIT) cluster_barrier();
        return;
    }

    // ---- the top values. A bound that at least `top` threads' maxima reach and not many more: bit by bit
    // from the first in which they differ, towards the top-th largest. With fewer threads than that, all
    // values are candidates.
    uint64_t bound = 0;
    if (tid == 0) n_groups = n_list = 0;
    if (max(min(NT, nvec), edge) >= top) {
        constexpr int kShift = 32 - 8 * sizeof(T);   // bf16: the lower half says nothing
        const uint32_t mine_order = has ? order(mine) >> kShift : 0, hi = order(m) >> kShift;
        const int bits = 32 - __clz(hi ^ (order(low) >> kShift));   // 0 when all are equal
        uint32_t b = bits == 32 ? 0 : hi >> bits << bits;
        for (int bit = bits - 1; bit >= 0; --bit) {
            const uint32_t cand = b | (1u << bit);
            const int count = __syncthreads_count(mine_order >= cand);
            if (count >= top) b = cand;
            if (count >= top && count <= top + top / 2 + 4) break;
        }
        if (kShift) b = b << 16 | (b >> 15 ? 0u : 0xFFFFu);
        bound = static_cast<uint64_t>(b) << 32;
    }
    __syncthreads();
    if (order(best) >= bound >> 32)   // no group holds more than its thread's largest, nor an upper half above its own
        for (int g = 0; g < n_mine; ++g) {
            if (group_max[g * NT + tid] < bound >> 48) continue;
            const int at = atomicAdd(&n_groups, 1);
            if (at < kGroups) groups[at] = g * A * NT + tid;   // its first vector
        }
    const Offers offers = {bound, list, &n_list};
    if (my_edge >= 0) offers.add(rank_key(ev, base + static_cast<uint32_t>(my_edge)));
    __syncthreads();
    if (n_groups <= kGroups) {
        for (int q = tid; q < n_groups * A; q += NT) {
            const int at = groups[q / A] + q % A * NT;
            if (at < nvec) offers.add_vector<T>(xv + at, base + static_cast<uint32_t>(head + at * E));
        }
    }
    __syncthreads();
    if (n_groups > kGroups || n_list > kList) {
        const Mine own = {xv, nvec, n_mine, best_group, base + static_cast<uint32_t>(head), order(best),
                          my_edge >= 0 ? rank_key(ev, base + static_cast<uint32_t>(my_edge)) : 0};
        second_look<T, NT, A>(own, group_max, top, list, &n_list, groups, &n_groups);
        if (n_list > kList) {   // more values from the bound up than the list holds
            if constexpr (SPLIT) {
                if (tid == 0) failed = 1;
            } else {
                careful_row<T, NT>(row, r, row_len, y, top, out, tmp64);
                return;
            }
        }
    }
    int n = min(n_list, kList);
    if constexpr (SPLIT) {   // the block's own top values, then those of all, by the row's first block
        for (int c = tid; c < n; c += NT) {
            int place = 0;
            for (int i = 0; i < n; ++i) place += list[i] > list[c];
            if (place < top) mine_top[place] = list[c];
        }
        cluster_barrier();
        if (rank == 0) {
            bool lost = false;
            for (int i = 0; i < parts; ++i) lost |= remote_u32(&failed, i) != 0;
            n = parts * top;
            if (tid < n) {   // parts * top <= 8 * 32
                const uint64_t* at = &mine_top[tid % top];
                list[tid] = remote_u32(at, tid / top) | static_cast<uint64_t>(remote_u32(reinterpret_cast<const uint32_t*>(at) + 1, tid / top)) << 32;
            }
            if (lost) {
                __syncthreads();
                careful_row<T, NT>(row, r, row_len, y, top, out, tmp64);
                n = 0;
            }
        }
        cluster_barrier();
        if (rank != 0) return;
    }
    for (int c = tid; c < n; c += NT) {
        const uint64_t key = list[c];
        int place = 0;
        for (int i = 0; i < n; ++i) place += list[i] > key;
        if (place < top && key && KQ_IN_RANGE(key_index(key), row_len)) {
            out.top_id[r * top + place] = static_cast<int32_t>(key_index(key));
            out.top_logp[r * top + place] = logp_of(key_value(key), r2, lz2);
        }
    }
}

template <typename T, int NT, bool SPLIT = false>
kq_status run_logprob(const T* logits, int64_t rows, int64_t V, int64_t ld, const int64_t* target, int top, const Out& out,
                      cudaStream_t stream, int parts = 1) {
    // runs of whole vectors, so that they all lie to 16 bytes as their row does
    const int64_t part = cdiv(cdiv(V, parts), 64) * 64;
    const int64_t group = (NT == kWide ? kWideAhead : kAhead) * NT * (16 / sizeof(T));   // values of a group of every thread
    static std::atomic<uint64_t> done{0};
    KQ_TRY(once_per_device(done, [&] {
        KQ_CUDA(cudaFuncSetAttribute(logprob_kernel<T, NT, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(cdiv(KQ_LOGPROBS_MAX_V, group) * NT * sizeof(uint16_t))));
        return KQ_OK;
    }));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(rows * parts));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = top ? static_cast<size_t>(cdiv(SPLIT ? part : V, group)) * NT * sizeof(uint16_t) : 0;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {static_cast<unsigned>(parts), 1, 1};
    cfg.attrs = at;
    cfg.numAttrs = SPLIT ? 1 : 0;
    KQ_CUDA(cudaLaunchKernelEx(&cfg, logprob_kernel<T, NT, SPLIT>, logits, V, ld, target, top, out, parts, static_cast<int>(part)));
    return KQ_OK;
}

template <typename T>
kq_status pick_logprob(const T* x, int64_t rows, int64_t V, int64_t ld, const int64_t* target, int top, const Out& out,
                       cudaStream_t stream) {
    const int64_t bytes = V * static_cast<int64_t>(sizeof(T));
    int parts = 1;   // blocks of a row, a power of two
    while (parts < kCluster && rows * parts * 2 <= num_sms() && bytes >= kSplitBytes * 2 * parts) parts *= 2;
    if (parts > 1) return run_logprob<T, kSplit, true>(x, rows, V, ld, target, top, out, stream, parts);
    if (bytes < kShortRow) return run_logprob<T, kNarrow>(x, rows, V, ld, target, top, out, stream);
    if (rows <= num_sms()) return run_logprob<T, kWide>(x, rows, V, ld, target, top, out, stream);
    if (rows <= 2 * num_sms()) return run_logprob<T, kSplit>(x, rows, V, ld, target, top, out, stream);
    if (bytes < kMiddleRow) return run_logprob<T, kMedium>(x, rows, V, ld, target, top, out, stream);
    return run_logprob<T, kThreads>(x, rows, V, ld, target, top, out, stream);
}

template <typename T>
struct Grad {
    const T* logits;
    T* grad;
    int64_t V, ld, ld_grad;
    const int64_t* target;
    const float *lse, *entropy, *g_logp, *g_entropy;
    int* info;
};

__device__ __forceinline__ float grad_of(float x, float sum, float g, float ge, float h) {
    const float lp = x - sum, p = ex2(lp * kLog2e);
    return p > 0.0f ? -p * fmaf(ge, lp + h, g) : p == p ? 0.0f : p;
}

// Blocks (row, part). VEC: logits and grad have the same place in 16 bytes, so a row is vectors with a few
// values before and after them; else one value at a time.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(const Grad<T> a) {
    constexpr int E = 16 / sizeof(T);
    const int64_t r = blockIdx.x;
    const T* x = a.logits + r * a.ld;
    T* d = a.grad + r * a.ld_grad;
    const int64_t y = a.target[r];
    if (y >= a.V && threadIdx.x == 0 && blockIdx.y == 0) record_error(a.info, -KQ_ERR_INVALID_ARG);
    const float sum = a.lse[r], g = y >= 0 && y < a.V ? a.g_logp[r] : 0.0f;
    const float ge = a.g_entropy ? a.g_entropy[r] : 0.0f, h = a.g_entropy ? a.entropy[r] : 0.0f;
    const bool none = sum == -INFINITY;
    auto one = [&](int64_t v) {
        const float q = none ? 0.0f : grad_of(value(x, v), sum, g, ge, h);
        if (KQ_IN_RANGE(v, a.V)) d[v] = static_cast<T>(v == y && !none ? q + g : q);
    };
    if constexpr (VEC) {
        const int64_t head = min(a.V, static_cast<int64_t>((16 - (reinterpret_cast<uintptr_t>(x) & 15)) % 16 / sizeof(T)));
        const int64_t n = (a.V - head) / E, tail = a.V - head - n * E;
        const uint4* xv = reinterpret_cast<const uint4*>(x + head);
        uint4* dv = reinterpret_cast<uint4*>(d + head);
        if (blockIdx.y == 0 && threadIdx.x < head + tail)
            one(threadIdx.x < head ? threadIdx.x : n * E + threadIdx.x);
        const int64_t ty = y >= head && !none ? (y - head) / E : -1;   // the target's vector
        const int64_t step = static_cast<int64_t>(gridDim.y) * kThreads * kAhead;
        for (int64_t j0 = static_cast<int64_t>(blockIdx.y) * kThreads * kAhead + threadIdx.x; j0 < n; j0 += step) {
            uint4 u[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (j0 + i * kThreads < n) u[i] = __ldcs(xv + j0 + i * kThreads);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t j = j0 + i * kThreads;
                if (j >= n) break;
                float q[E];
                const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    const uint32_t b = sizeof(T) == 4 ? w[k % 4] : k & 1 ? w[k / 2] & 0xFFFF0000u : w[k / 2] << 16;
                    q[k] = none ? 0.0f : grad_of(__uint_as_float(b), sum, g, ge, h);
                }
                if (j == ty) {
#pragma unroll
                    for (int k = 0; k < E; ++k)
                        if (head + j * E + k == y) q[k] += g;
                }
                uint4 o;
                if constexpr (sizeof(T) == 4) {
                    o = make_uint4(__float_as_uint(q[0]), __float_as_uint(q[1]), __float_as_uint(q[2]), __float_as_uint(q[3]));
                } else {
                    uint32_t b[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const __nv_bfloat162 t = __floats2bfloat162_rn(q[2 * k], q[2 * k + 1]);
                        b[k] = *reinterpret_cast<const uint32_t*>(&t);
                    }
                    o = make_uint4(b[0], b[1], b[2], b[3]);
                }
                if (KQ_IN_RANGE(head + j * E + E - 1, a.V)) __stcs(dv + j, o);
            }
        }
    } else {
        for (int64_t v = static_cast<int64_t>(blockIdx.y) * kThreads + threadIdx.x; v < a.V;
             v += static_cast<int64_t>(gridDim.y) * kThreads)
            one(v);
    }
}

template <typename T>
kq_status run_grad(const Grad<T>& a, int64_t rows, cudaStream_t stream) {
    const bool vec = !((reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.grad)) & 15u) &&
                     !(((a.ld - a.ld_grad) * sizeof(T)) & 15u);
    // a row to a block, cut in parts of at least one round of its threads while there are few rows
    const int64_t rounds = cdiv(a.V, vec ? 16 / sizeof(T) * kThreads * kAhead : kThreads);
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(rounds, cdiv(static_cast<int64_t>(num_sms()) * 16, rows)));
    const dim3 grid(static_cast<unsigned>(rows), static_cast<unsigned>(std::min<int64_t>(parts, 65535)));
    if (vec) logprob_grad_kernel<T, true><<<grid, kThreads, 0, stream>>>(a);
    else logprob_grad_kernel<T, false><<<grid, kThreads, 0, stream>>>(a);
    KQ_LAUNCH_CHECK("logprob_grad_kernel");
    return KQ_OK;
}

}  // namespace

KQ_DEBUG_UNIT(logprob)
}  // namespace kq

using namespace kq;

namespace {
bool bad_logits(const char* who, const void* logits, int dtype, int64_t T, int64_t V, int64_t ld, kq_status* st) {
    *st = KQ_OK;
    if (dtype != KQ_BF16 && dtype != KQ_F32) {
        set_error("%s: dtype must be KQ_BF16 or KQ_F32", who);
        *st = KQ_ERR_UNSUPPORTED;
    } else if (V > KQ_LOGPROBS_MAX_V) {
        set_error("%s: V must be at most %d", who, KQ_LOGPROBS_MAX_V);
        *st = KQ_ERR_UNSUPPORTED;
    } else if (T < 0 || T > 0x7fffffffll || V < 1 || ld < V || (T > 0 && !logits) ||
               (reinterpret_cast<uintptr_t>(logits) & (dtype == KQ_BF16 ? 1u : 3u))) {
        set_error("%s: 0 <= T < 2^31, V >= 1, ld >= V and aligned logits needed", who);
        *st = KQ_ERR_INVALID_ARG;
    }
    return *st != KQ_OK;
}
}  // namespace

extern "C" kq_status kq_token_logprobs(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                                       const int64_t* target, int top, float* logp, float* entropy, float* lse,
                                       int32_t* top_id, float* top_logp, int* info, kq_stream_t stream_) {
    kq_status st;
    if (bad_logits("kq_token_logprobs", logits, dtype, T, V, ld, &st)) return st;
    if (top < 0 || top > KQ_LOGPROBS_MAX_TOP || top > V || (T > 0 && (!target || !logp || (top > 0 && (!top_id || !top_logp))))) {
        set_error("kq_token_logprobs: target and logp must not be NULL, 0 <= top <= min(%d, V) with top_id and top_logp",
                  KQ_LOGPROBS_MAX_TOP);
        return KQ_ERR_INVALID_ARG;
    }
    if (T == 0) return KQ_OK;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    const Out out = {logp, entropy, lse, top_id, top_logp, info};
    // A row's joint steps take a block about as long as half a large row's values: many small blocks on an SM
    // cover them for each other, the smaller the shorter the row (V = 32000 bf16: 128 threads 202 us, 256 226 us;
    // V = 128000: 216 and 190 us; V = 4000: 64 threads 69 us, 128 78 us, 256 120 us, each 16384 rows but 4096
    // of the largest); blocks alone or in
    // twos on an SM are shorter with more threads (300 rows of 128000 bf16 27 us with 1024, 20 us with 512), and a few rows
    // with a cluster each (8 rows: 12.3 us with one block a row, 10.3 us with eight).
    const kq_status launched =
        dtype == KQ_BF16 ? pick_logprob(static_cast<const __nv_bfloat16*>(logits), T, V, ld, target, top, out, stream)
                         : pick_logprob(static_cast<const float*>(logits), T, V, ld, target, top, out, stream);
    KQ_TRY(launched);
    KQ_LAUNCH_CHECK("logprob_kernel");
    return KQ_OK;
}

extern "C" kq_status kq_token_logprobs_grad(const void* logits, int dtype, int64_t T, int64_t V, int64_t ld,
                                            const int64_t* target, const float* lse, const float* entropy,
                                            const float* g_logp, const float* g_entropy, void* grad, int64_t ld_grad,
                                            int* info, kq_stream_t stream_) {
    kq_status st;
    if (bad_logits("kq_token_logprobs_grad", logits, dtype, T, V, ld, &st)) return st;
    if ((T > 0 && (!target || !lse || !g_logp || !grad || (g_entropy && !entropy))) || ld_grad < V ||
        (grad == logits && ld_grad != ld) || (reinterpret_cast<uintptr_t>(grad) & (dtype == KQ_BF16 ? 1u : 3u))) {
        set_error("kq_token_logprobs_grad: target, lse, g_logp, grad (and entropy with g_entropy) must not be NULL, ld_grad "
                  ">= V, and ld_grad = ld in place");
        return KQ_ERR_INVALID_ARG;
    }
    if (T == 0) return KQ_OK;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (dtype == KQ_BF16)
        return run_grad(Grad<__nv_bfloat16>{static_cast<const __nv_bfloat16*>(logits), static_cast<__nv_bfloat16*>(grad), V, ld,
                                            ld_grad, target, lse, entropy, g_logp, g_entropy, info}, T, stream);
    return run_grad(Grad<float>{static_cast<const float*>(logits), static_cast<float*>(grad), V, ld, ld_grad, target, lse, entropy,
                                g_logp, g_entropy, info}, T, stream);
}
