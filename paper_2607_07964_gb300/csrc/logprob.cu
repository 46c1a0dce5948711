// kq_token_logprobs and its gradient. One block for a row: the maximum, then the sum of e^(x - m)
// and of e^(x - m) (m - x), then the top tokens one after the other, each the largest below the one
// before in the order (logit descending, index ascending).
//   entropy = ln Z + sum e^(x - m) (m - x) / Z: both terms are at least 0, so nothing cancels.
#include <algorithm>

#include "kv_common.cuh"

namespace kq {
namespace {

constexpr int kThreads = 512;

__device__ __forceinline__ float value(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float value(const __nv_bfloat16* p, int64_t i) { return __bfloat162float(p[i]); }

// Larger for a larger logit, then for a smaller index; NaN above every number.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t i) {
    uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    u = isnan(x) ? 0xFFFFFFFFu : (u >> 31) ? ~u : (u | 0x80000000u);
    return (static_cast<uint64_t>(u) << 32) | (0xFFFFFFFFu - i);
}

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* tmp, F f) {
    for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = v;
    __syncthreads();
    v = tmp[0];
    for (int i = 1; i < kThreads / 32; ++i) v = f(v, tmp[i]);
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_kernel(const T* __restrict__ logits, int64_t V, int64_t ld,
                                                           const int64_t* __restrict__ target, int top,
                                                           float* __restrict__ logp, float* __restrict__ entropy,
                                                           float* __restrict__ lse, int32_t* __restrict__ top_id,
                                                           float* __restrict__ top_logp, int* info) {
    __shared__ uint64_t tmp64[kThreads / 32];
    float* tmp = reinterpret_cast<float*>(tmp64);
    const int64_t r = blockIdx.x;
    const T* x = logits + r * ld;
    float m = -INFINITY;
    bool bad = false;
    for (int64_t i = threadIdx.x; i < V; i += kThreads) {
        const float v = value(x, i);
        bad |= isnan(v) || v == INFINITY;
        m = fmaxf(m, v);
    }
    m = block_reduce(m, tmp, [](float a, float b) { return fmaxf(a, b); });
    bad = __syncthreads_or(bad);
    float z = 0.0f, w = 0.0f;
    for (int64_t i = threadIdx.x; i < V; i += kThreads) {
        const float d = value(x, i) - m;
        if (d > -INFINITY) {
            const float e = expf(d);
            z += e;
            w -= e * d;
        }
    }
    z = block_reduce(z, tmp, [](float a, float b) { return a + b; });
    w = block_reduce(w, tmp, [](float a, float b) { return a + b; });
    const float lz = logf(z);
    const bool none = m == -INFINITY;
    const float sum = bad ? NAN : none ? -INFINITY : m + lz;
    if (threadIdx.x == 0) {
        const int64_t y = target[r];
        float lp = 0.0f;
        if (y >= V) {
            record_error(info, -KQ_ERR_INVALID_ARG);
            lp = NAN;
        } else if (y >= 0) {
            lp = bad ? NAN : none ? -INFINITY : value(x, y) - m - lz;
        }
        logp[r] = lp;
        if (entropy) entropy[r] = bad ? NAN : none ? 0.0f : lz + w / z;
        if (lse) lse[r] = sum;
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t best = 0;
        for (int64_t i = threadIdx.x; i < V; i += kThreads) {
            const uint64_t key = rank_key(value(x, i), static_cast<uint32_t>(i));
            if (key < last && key > best) best = key;
        }
        best = block_reduce(best, tmp64, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
        last = best;
        if (threadIdx.x == 0) {
            const int64_t i = 0xFFFFFFFFu - static_cast<uint32_t>(best);
            top_id[r * top + k] = static_cast<int32_t>(i);
            top_logp[r * top + k] = bad ? NAN : none ? -INFINITY : value(x, i) - m - lz;
        }
    }
}

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(const T* logits, int64_t V, int64_t ld,
                                                                const int64_t* __restrict__ target,
                                                                const float* __restrict__ lse,
                                                                const float* __restrict__ entropy,
                                                                const float* __restrict__ g_logp,
                                                                const float* __restrict__ g_entropy, T* grad,
                                                                int64_t ld_grad, int* info) {
    const int64_t r = blockIdx.x;
    const int64_t y = target[r];
    if (y >= V && threadIdx.x == 0) record_error(info, -KQ_ERR_INVALID_ARG);
    const float g = y >= 0 && y < V ? g_logp[r] : 0.0f;
    const float ge = g_entropy ? g_entropy[r] : 0.0f, h = g_entropy ? entropy[r] : 0.0f, sum = lse[r];
    for (int64_t i = threadIdx.x; i < V; i += kThreads) {
        const float v = value(logits + r * ld, i);
        float d = 0.0f;
        if (sum != -INFINITY) {
            const float lp = v - sum, p = expf(lp);
            d = -g * p;
            if (g_entropy && p != 0.0f) d -= ge * p * (lp + h);
            if (i == y) d += g;
        }
        put(grad + r * ld_grad + i, d);
    }
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
    if (dtype == KQ_BF16)
        logprob_kernel<<<static_cast<unsigned>(T), kThreads, 0, stream>>>(static_cast<const __nv_bfloat16*>(logits), V, ld, target,
                                                                        top, logp, entropy, lse, top_id, top_logp, info);
    else
        logprob_kernel<<<static_cast<unsigned>(T), kThreads, 0, stream>>>(static_cast<const float*>(logits), V, ld, target, top,
                                                                        logp, entropy, lse, top_id, top_logp, info);
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
        logprob_grad_kernel<<<static_cast<unsigned>(T), kThreads, 0, stream>>>(
            static_cast<const __nv_bfloat16*>(logits), V, ld, target, lse, entropy, g_logp, g_entropy,
            static_cast<__nv_bfloat16*>(grad), ld_grad, info);
    else
        logprob_grad_kernel<<<static_cast<unsigned>(T), kThreads, 0, stream>>>(static_cast<const float*>(logits), V, ld, target, lse,
                                                                             entropy, g_logp, g_entropy,
                                                                             static_cast<float*>(grad), ld_grad, info);
    KQ_LAUNCH_CHECK("logprob_grad_kernel");
    return KQ_OK;
}
