// kq_kv_attend: attention over the 4-bit cache. One block for a token and query head: tiles of
// 128 slots, a thread a slot for the scores, a thread a dimension for the sum of values, with the
// running maximum and sum of an online softmax. The weights of the slots come from the stored
// scores and the finished log-sum in a second kernel.
#include <algorithm>

#include "kv_common.cuh"

namespace kq {
namespace {

constexpr int kTile = 128;

__device__ __forceinline__ int64_t visible(const int32_t* start, int b, int64_t i, int64_t n) {
    const int64_t m = n - (start[b + 1] - 1 - i);
    return m < 0 ? 0 : m;
}

template <typename T, int D>
__global__ void __launch_bounds__(kTile) kv_attend_kernel(KvView c, const T* __restrict__ q, int64_t tokens, int q_heads,
                                                          int64_t ts, int64_t hs, const int32_t* __restrict__ start,
                                                          const int32_t* __restrict__ lens, float scale, T* __restrict__ out,
                                                          float* __restrict__ lse, float* __restrict__ scores, int64_t S,
                                                          int* info) {
    __shared__ float qs[D], p[kTile], red[4];
    __shared__ const uint8_t* gran[kTile / kGranule];
    if (blockIdx.x == 0 && threadIdx.x == 0 && (start[0] != 0 || start[c.batch] != tokens)) record_error(info, -KQ_ERR_INVALID_ARG);
    const int64_t i = blockIdx.x / q_heads;
    const int hq = static_cast<int>(blockIdx.x % q_heads);
    const int group = q_heads / c.kv_heads, h = hq / group, tid = threadIdx.x;
    const int b = kv_sequence_of(start, c.batch, i);
    if (b < 0) {
        record_error(info, -KQ_ERR_INVALID_ARG);
        return;
    }
    const int64_t cap = scores ? min(kv_capacity(c), S) : kv_capacity(c);
    const int64_t n = visible(start, b, i, kv_length(lens, b, cap, info));
    for (int d = tid; d < D; d += kTile) qs[d] = static_cast<float>(q[i * ts + hq * hs + d]) * scale;
    float m = -INFINITY, z = 0.0f, o = 0.0f;
    for (int64_t base = 0; base < n; base += kTile) {
        __syncthreads();
        if (tid < kTile / kGranule) {
            const int64_t s0 = base + tid * kGranule;
            const uint8_t* g = s0 < n ? kv_granule(c, b, h, s0) : c.data;
            if (!g) record_error(info, -KQ_ERR_INVALID_ARG);
            gran[tid] = g ? g : c.data;
        }
        __syncthreads();
        float s = -INFINITY;
        if (base + tid < n) {
            const uint8_t* g = gran[tid / kGranule];
            const uint8_t* row = g + kv_code_at(D, 0, tid % kGranule);
            const uint32_t prm = *reinterpret_cast<const uint32_t*>(g + kv_param_at(D, 0, tid % kGranule));
            s = 0.0f;
            for (int d = 0; d < D; ++d)
                s = fmaf(qs[d], fmaf(kv_scale(prm), static_cast<float>((row[d / 2] >> (4 * (d & 1))) & 15), kv_offset(prm)), s);
            if (scores) scores[((i * c.kv_heads + h) * S + base + tid) * group + hq % group] = s;
        }
        float w = s;
        for (int off = 16; off > 0; off >>= 1) w = fmaxf(w, __shfl_xor_sync(0xffffffffu, w, off));
        if (isnan(s)) w = s;
        if ((tid & 31) == 0) red[tid >> 5] = w;
        __syncthreads();
        const float mn = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
        p[tid] = s == -INFINITY ? 0.0f : expf(s - mn);
        __syncthreads();
        const float r = m == -INFINITY ? 0.0f : expf(m - mn);
        m = mn;
        z *= r;
        o *= r;
        const int many = static_cast<int>(min(static_cast<int64_t>(kTile), n - base));
        for (int t = 0; t < many; ++t) {
            z += p[t];
            if (tid < D) {
                const uint8_t* g = gran[t / kGranule];
                const uint32_t prm = *reinterpret_cast<const uint32_t*>(g + kv_param_at(D, 1, t % kGranule));
                const int code = (g[kv_code_at(D, 1, t % kGranule) + tid / 2] >> (4 * (tid & 1))) & 15;
                o = fmaf(p[t], fmaf(kv_scale(prm), static_cast<float>(code), kv_offset(prm)), o);
            }
        }
    }
    if (tid < D) out[(i * q_heads + hq) * D + tid] = static_cast<T>(n > 0 ? o / z : 0.0f);
    if (tid == 0 && lse) lse[i * q_heads + hq] = n > 0 ? m + logf(z) : -INFINITY;
}

__global__ void kv_weight_kernel(KvView c, int q_heads, const int32_t* __restrict__ start, const int32_t* __restrict__ lens,
                                 const float* __restrict__ scores, const float* __restrict__ lse, float* __restrict__ acc,
                                 int64_t S) {
    const int b = blockIdx.y / c.kv_heads, h = blockIdx.y % c.kv_heads, group = q_heads / c.kv_heads;
    const int64_t slot = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    const int64_t n = kv_length(lens, b, min(kv_capacity(c), S), nullptr);
    if (slot >= n) return;
    float sum = 0.0f;
    for (int64_t i = start[b]; i < start[b + 1]; ++i) {
        if (slot >= visible(start, b, i, n)) continue;
        for (int g = 0; g < group; ++g)
            sum += expf(scores[((i * c.kv_heads + h) * S + slot) * group + g] - lse[i * q_heads + h * group + g]);
    }
    acc[(static_cast<int64_t>(b) * c.kv_heads + h) * S + slot] += sum;
}

}  // namespace

KQ_DEBUG_UNIT(kv_attend)
}  // namespace kq

using namespace kq;

extern "C" size_t kq_kv_attend_workspace(int64_t T, int64_t q_heads, int64_t kv_heads, int64_t dim, int64_t S) {
    if (T < 1 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || dim < 1 || S < 0) return 0;
    return S ? static_cast<size_t>(T) * q_heads * (S + 64) * sizeof(float) : 0;
}

extern "C" kq_status kq_kv_attend(const kq_kv_cache* cache, const void* q, int dtype, int64_t T, int64_t q_heads,
                                  int64_t q_token_stride, int64_t q_head_stride, const int32_t* start,
                                  const int32_t* lens, float scale, void* out, float* lse, float* acc, int64_t S, int* info,
                                  void* ws, size_t ws_bytes, kq_stream_t stream_) {
    KvView c;
    KQ_TRY(kv_view(cache, "kq_kv_attend", &c));
    if (dtype != KQ_BF16 && dtype != KQ_F32) {
        set_error("kq_kv_attend: dtype must be KQ_BF16 or KQ_F32");
        return KQ_ERR_UNSUPPORTED;
    }
    const uintptr_t es = dtype == KQ_BF16 ? 2 : 4;
    if (T < 0 || T > 0x7fffffffll || q_heads < 1 || q_heads % c.kv_heads || !start || !lens || (T > 0 && (!q || !out)) ||
        (acc && S < 1) || !(scale - scale == 0.0f) ||
        ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & (es - 1))) {
        set_error("kq_kv_attend: q, out, start, lens must not be NULL, q_heads a multiple of kv_heads, scale finite, "
                  "S >= 1 with acc");
        return KQ_ERR_INVALID_ARG;
    }
    if (T == 0) return KQ_OK;
    const size_t need = kq_kv_attend_workspace(T, q_heads, c.kv_heads, c.dim, acc ? S : 0);
    if (need && (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u))) {
        set_error("kq_kv_attend: workspace must be 256-byte aligned and hold %zu bytes", need);
        return KQ_ERR_WORKSPACE;
    }
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    float* scores = acc ? static_cast<float*>(ws) : nullptr;
    float* sums = lse;
    if (acc && !lse) sums = scores + static_cast<size_t>(T) * q_heads * S;
    const unsigned grid = static_cast<unsigned>(T * q_heads);
#define KQ_ATTEND(TY, DIM)                                                                                         \
    kv_attend_kernel<TY, DIM><<<grid, kTile, 0, stream>>>(c, static_cast<const TY*>(q), T, static_cast<int>(q_heads), \
                                                          q_token_stride, q_head_stride, start, lens, scale,       \
                                                          static_cast<TY*>(out), sums, scores, S, info)
    if (dtype == KQ_BF16) c.dim == 128 ? KQ_ATTEND(__nv_bfloat16, 128) : KQ_ATTEND(__nv_bfloat16, 64);
    else c.dim == 128 ? KQ_ATTEND(float, 128) : KQ_ATTEND(float, 64);
#undef KQ_ATTEND
    KQ_LAUNCH_CHECK("kv_attend_kernel");
    if (acc) {
        const dim3 wg(static_cast<unsigned>(cdiv(std::min<int64_t>(S, kv_capacity(c)), 256)),
                      static_cast<unsigned>(c.batch * c.kv_heads));
        kv_weight_kernel<<<wg, 256, 0, stream>>>(c, static_cast<int>(q_heads), start, lens, scores, sums, acc, S);
        KQ_LAUNCH_CHECK("kv_weight_kernel");
    }
    return KQ_OK;
}
