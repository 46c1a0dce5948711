// kq_kv_append and kq_kv_read: rows of keys and values into the 4-bit cache and back.
//
// A row is D values of one token and head. o = min(x) rounded down to bf16, s = (max(x) - o) / 15
// rounded up to bf16, c = rint((x - o) / s): with o below every value and s at least a fifteenth
// of the range above it no code needs clamping, so the error is at most s / 2 everywhere. The
// rounding of s costs at most 2^-8 of the step, in exchange for 4 bytes of parameters a row
// instead of 8 (D = 128: 68 bytes a row, 4.25 bits a value).
//
// Both are bound by memory: append reads 2 D e and writes D + 8 bytes for each token and head
// (e bytes a value), read the reverse. D / 8 lanes take a row, 8 values each, which is one 16-byte
// load of bf16 (two of fp32) and one 4-byte word of codes; the minimum and maximum go through
// shuffles inside those lanes, so nothing is staged.
#include <algorithm>

#include "kv_common.cuh"

namespace kq {

kq_status kv_view(const kq_kv_cache* c, const char* who, KvView* v) {
    if (!c || !c->data || !c->table) {
        set_error("%s: cache, its data and its table must not be NULL", who);
        return KQ_ERR_INVALID_ARG;
    }
    if (c->dim != 64 && c->dim != 128) {
        set_error("%s: dim must be 64 or 128, got %lld", who, (long long)c->dim);
        return KQ_ERR_UNSUPPORTED;
    }
    if (c->page < kGranule || c->page > 1024 || c->page % kGranule || c->pages < 1 || c->pages > 0x7fffffffll ||
        c->kv_heads < 1 || c->kv_heads > 65535 || c->batch < 1 || c->batch > 65535 || c->batch * c->kv_heads > (1 << 24) ||
        c->table_ld < 1 || c->table_ld > 0x7fffffffll ||
        c->table_ld * c->page > 0x7fffffffll - 1024 || (reinterpret_cast<uintptr_t>(c->data) & 15u)) {
        set_error("%s: page must be a multiple of 16 up to 1024, pages, kv_heads, batch and table_ld in range, data "
                  "16-byte aligned", who);
        return KQ_ERR_INVALID_ARG;
    }
    v->data = c->data;
    v->table = c->table;
    v->pages = c->pages;
    v->page = static_cast<int32_t>(c->page);
    v->kv_heads = static_cast<int32_t>(c->kv_heads);
    v->dim = static_cast<int32_t>(c->dim);
    v->batch = static_cast<int32_t>(c->batch);
    v->table_ld = c->table_ld;
    return KQ_OK;
}

namespace {

constexpr int kThreads = 256;

// 8 consecutive values. VEC: 16-byte loads (the caller checked base and strides).
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
    if constexpr (VEC && sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else if constexpr (VEC) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(p[i]);
    }
}

struct RowSource {
    const void* p[2];               // k, v
    int64_t token[2], head[2];      // strides in elements
};

// One row per D / 8 lanes; rows are ordered (token, head, key then value).
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(KvView c, RowSource src, int64_t tokens,
                                                             const int32_t* __restrict__ start,
                                                             const int32_t* __restrict__ lens, int32_t* lens_out,
                                                             float* __restrict__ acc, int32_t* __restrict__ pos, int64_t S,
                                                             const int32_t* __restrict__ seen, int32_t* seen_out, int* info) {
    constexpr int kLanes = D / 8;
    const int64_t tid = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t cap = kv_capacity(c);
    if (blockIdx.x == 0) {
        for (int b = threadIdx.x; b < c.batch; b += kThreads) {
            const int64_t add = max(0, start[b + 1] - start[b]);
            const int64_t n = kv_length(lens, b, cap, info);
            if (n + add > cap) record_error(info, -KQ_ERR_INVALID_ARG);
            if (lens_out) lens_out[b] = static_cast<int32_t>(min(n + add, cap));
            if (seen_out) seen_out[b] = static_cast<int32_t>((seen ? seen[b] : n) + add);
        }
        if (threadIdx.x == 0 && (start[0] != 0 || start[c.batch] != tokens)) record_error(info, -KQ_ERR_INVALID_ARG);
    }
    const int lane = threadIdx.x % kLanes;
    const uint32_t mask = (kLanes == 16 ? 0xFFFFu : 0xFFu) << (threadIdx.x % 32 - lane);
    const int64_t rows = tokens * c.kv_heads * 2;
    for (int64_t row = tid / kLanes; row < rows; row += static_cast<int64_t>(gridDim.x) * (kThreads / kLanes)) {
        const int which = static_cast<int>(row & 1);
        const int h = static_cast<int>((row >> 1) % c.kv_heads);
        const int64_t i = (row >> 1) / c.kv_heads;
        const int b = kv_sequence_of(start, c.batch, i);
        if (b < 0) continue;   // uniform over the row's lanes; recorded by the first block
        const int64_t n = kv_length(lens, b, cap, info);
        const int64_t slot = n + (i - start[b]);
        uint8_t* g = slot < cap ? kv_granule(c, b, h, slot) : nullptr;
        if (!g) {
            record_error(info, -KQ_ERR_INVALID_ARG);
            continue;
        }
        const T* p = static_cast<const T*>(src.p[which]) + i * src.token[which] + h * src.head[which] + lane * 8;
        float x[8];
        load8<T, VEC>(p, x);
        float lo = x[0], hi = x[0];
        bool fine = true;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            lo = fminf(lo, x[k]);
            hi = fmaxf(hi, x[k]);
            fine &= fabsf(x[k]) <= 3.402823466e38f;   // false for NaN as well
        }
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) {
            lo = fminf(lo, __shfl_xor_sync(mask, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(mask, hi, o));
        }
        fine = __all_sync(mask, fine);
        // down to bf16: negative values get a larger magnitude; up to bf16: the scale is >= 0
        const uint32_t lb = __float_as_uint(lo);
        const uint32_t ob = (lb + ((lb >> 31) ? 0xFFFFu : 0u)) & 0xFFFF0000u;
        const float off = __uint_as_float(ob);
        const uint32_t sb = (__float_as_uint(__fdiv_rn(__fsub_rn(hi, off), 15.0f)) + 0xFFFFu) & 0xFFFF0000u;
        const float s = __uint_as_float(sb);
        fine = fine && isfinite(off) && isfinite(s);
        uint32_t word = 0;
        if (fine && s > 0.0f) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float q = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[k], off), s)), 0.0f), 15.0f);
                word |= static_cast<uint32_t>(q) << (4 * k);
            }
        }
        const int t = static_cast<int>(slot % kGranule);
        reinterpret_cast<uint32_t*>(g + kv_code_at(D, which, t))[lane] = word;
        if (lane == 0) {
            *reinterpret_cast<uint32_t*>(g + kv_param_at(D, which, t)) = fine ? (sb >> 16) | ob : 0x7FC07FC0u;
            if (which == 0 && (acc || pos)) {
                if (slot < S) {
                    const int64_t at = (static_cast<int64_t>(b) * c.kv_heads + h) * S + slot;
                    if (acc) acc[at] = 0.0f;
                    if (pos) pos[at] = static_cast<int32_t>((seen ? seen[b] : n) + (i - start[b]));
                } else {
                    record_error(info, -KQ_ERR_INVALID_ARG);
                }
            }
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(KvView c, const int32_t* __restrict__ start,
                                                           const int32_t* __restrict__ first,
                                                           const int32_t* __restrict__ lens, int64_t tokens,
                                                           T* __restrict__ k, T* __restrict__ v, int* info) {
    constexpr int kLanes = D / 8;
    const int64_t tid = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int lane = threadIdx.x % kLanes;
    const int64_t cap = kv_capacity(c);
    const int64_t rows = tokens * c.kv_heads * 2;
    for (int64_t row = tid / kLanes; row < rows; row += static_cast<int64_t>(gridDim.x) * (kThreads / kLanes)) {
        const int which = static_cast<int>(row & 1);
        const int h = static_cast<int>((row >> 1) % c.kv_heads);
        const int64_t i = (row >> 1) / c.kv_heads;
        const int b = kv_sequence_of(start, c.batch, i);
        const uint8_t* g = nullptr;
        int64_t slot = 0;
        if (b >= 0) {
            slot = (first ? first[b] : 0) + (i - start[b]);
            const int64_t n = lens ? kv_length(lens, b, cap, info) : cap;
            if (slot < 0) record_error(info, -KQ_ERR_INVALID_ARG);
            if (slot >= 0 && slot < n) {
                g = kv_granule(c, b, h, slot);
                if (!g) record_error(info, -KQ_ERR_INVALID_ARG);
            }
        }
        float x[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (g) {
            const int t = static_cast<int>(slot % kGranule);
            const uint32_t word = reinterpret_cast<const uint32_t*>(g + kv_code_at(D, which, t))[lane];
            const uint32_t prm = *reinterpret_cast<const uint32_t*>(g + kv_param_at(D, which, t));
            const float s = kv_scale(prm), off = kv_offset(prm);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(s, static_cast<float>((word >> (4 * j)) & 15u), off);
        }
        T* out = (which ? v : k) + (i * c.kv_heads + h) * D + lane * 8;
        if constexpr (sizeof(T) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
                w[j] = *reinterpret_cast<const uint32_t*>(&p);
            }
            *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            reinterpret_cast<float4*>(out)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(out)[1] = make_float4(x[4], x[5], x[6], x[7]);
        }
    }
}

int64_t row_blocks(int64_t rows, int dim) {
    return std::max<int64_t>(1, std::min<int64_t>(cdiv(rows * (dim / 8), kThreads), static_cast<int64_t>(num_sms()) * 32));
}

}  // namespace

KQ_DEBUG_UNIT(kv_store)
}  // namespace kq

using namespace kq;

extern "C" kq_status kq_kv_append(const kq_kv_cache* cache, const void* k, const void* v, int dtype, int64_t T,
                                  int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                                  int64_t v_head_stride, const int32_t* start, const int32_t* lens, int32_t* lens_out,
                                  float* acc, int32_t* pos, int64_t S, const int32_t* seen, int32_t* seen_out, int* info,
                                  kq_stream_t stream_) {
    KvView c;
    KQ_TRY(kv_view(cache, "kq_kv_append", &c));
    if (dtype != KQ_BF16 && dtype != KQ_F32) {
        set_error("kq_kv_append: dtype must be KQ_BF16 or KQ_F32");
        return KQ_ERR_UNSUPPORTED;
    }
    const uintptr_t es = dtype == KQ_BF16 ? 2 : 4;
    if (T < 0 || T > 0x7fffffffll || !start || !lens || (T > 0 && (!k || !v)) || ((acc || pos) && S < 1) ||
        lens_out == lens || (seen_out && seen_out == seen) || (lens_out && lens_out == seen_out) ||
        ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & (es - 1))) {
        set_error("kq_kv_append: start, lens, k, v must not be NULL, 0 <= T < 2^31, S >= 1 with acc or pos, lens_out and "
                  "seen_out apart from lens and seen");
        return KQ_ERR_INVALID_ARG;
    }
    RowSource src = {{k, v}, {k_token_stride, v_token_stride}, {k_head_stride, v_head_stride}};
    bool vec = true;
    for (int w = 0; w < 2; ++w)
        vec = vec && !(reinterpret_cast<uintptr_t>(src.p[w]) & 15u) && !((src.token[w] * es) & 15u) && !((src.head[w] * es) & 15u);
    const unsigned grid = static_cast<unsigned>(row_blocks(T * c.kv_heads * 2, c.dim));
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
#define KQ_APPEND(TY, DIM, VEC) \
    kv_append_kernel<TY, DIM, VEC><<<grid, kThreads, 0, stream>>>(c, src, T, start, lens, lens_out, acc, pos, S, seen, seen_out, info)
    if (dtype == KQ_BF16) {
        if (c.dim == 128) vec ? KQ_APPEND(__nv_bfloat16, 128, true) : KQ_APPEND(__nv_bfloat16, 128, false);
        else vec ? KQ_APPEND(__nv_bfloat16, 64, true) : KQ_APPEND(__nv_bfloat16, 64, false);
    } else {
        if (c.dim == 128) vec ? KQ_APPEND(float, 128, true) : KQ_APPEND(float, 128, false);
        else vec ? KQ_APPEND(float, 64, true) : KQ_APPEND(float, 64, false);
    }
#undef KQ_APPEND
    KQ_LAUNCH_CHECK("kv_append_kernel");
    return KQ_OK;
}

extern "C" kq_status kq_kv_read(const kq_kv_cache* cache, const int32_t* start, const int32_t* first,
                                const int32_t* lens, int dtype, int64_t T, void* k, void* v, int* info,
                                kq_stream_t stream_) {
    KvView c;
    KQ_TRY(kv_view(cache, "kq_kv_read", &c));
    if (dtype != KQ_BF16 && dtype != KQ_F32) {
        set_error("kq_kv_read: dtype must be KQ_BF16 or KQ_F32");
        return KQ_ERR_UNSUPPORTED;
    }
    if (T < 0 || T > 0x7fffffffll || !start || (T > 0 && (!k || !v)) ||
        ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)) {
        set_error("kq_kv_read: start, k, v must not be NULL, k and v 16-byte aligned, 0 <= T < 2^31");
        return KQ_ERR_INVALID_ARG;
    }
    if (T == 0) return KQ_OK;
    const unsigned grid = static_cast<unsigned>(row_blocks(T * c.kv_heads * 2, c.dim));
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
#define KQ_READ(TY, DIM)                                                                                         \
    kv_read_kernel<TY, DIM><<<grid, kThreads, 0, stream>>>(c, start, first, lens, T, static_cast<TY*>(k), \
                                                           static_cast<TY*>(v), info)
    if (dtype == KQ_BF16) c.dim == 128 ? KQ_READ(__nv_bfloat16, 128) : KQ_READ(__nv_bfloat16, 64);
    else c.dim == 128 ? KQ_READ(float, 128) : KQ_READ(float, 64);
#undef KQ_READ
    KQ_LAUNCH_CHECK("kv_read_kernel");
    return KQ_OK;
}
