// kq_kv_append and kq_kv_read: rows of keys and values into the 4-bit cache and back.
//
// A row is D values of one token and head. o = min(x) rounded down to bf16, s = (max(x) - o) / 15
// rounded up to bf16, c = rint((x - o) / s): with o below every value and s at least a fifteenth
// of the range above it no code needs clamping, so the error is at most s / 2 everywhere. The
// rounding of s costs at most 2^-8 of the step, in exchange for 4 bytes of parameters a row
// instead of 8 (D = 128: 68 bytes a row, 4.25 bits a value).
//
// Append reads 2 D e and writes D + 8 bytes for each token and head (e bytes a value), read the reverse. To
// append, a warp takes 8 consecutive tokens and, one after the other, the key and value rows of a few heads: a token's
// sequence, slot and page are looked up once for all of them, 8 parameters or positions fill a sector, and few heads
// leave no lane idle (a warp to a token with its heads side by side: 41 instead of 14 us for 51k tokens of one head, 43
// instead of 35 for four). Four lanes take a row, so that what a row costs once (two bounds, a division, a
// reciprocal) is shared by 32 values of a lane. 51k tokens of 8 heads, D = 128, take 58 us in bf16 (0.69 of the measured
// copy rate; bound by instructions and the latency of the loads) and 81 us in fp32 (0.88). Copying the
// rows ahead into shared memory was slower (82 and 125 us), prefetching them into L2 no faster. To read, a
// warp takes a token (of one or two heads, several) and D / 8 lanes a row, a word of codes each, as there is nothing to share.
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

// 16 consecutive values as they are loaded. VEC: 16 bytes at a time (the caller checked base and strides; 32 at a
// time were 1 to 2 us slower for 51k tokens of 8 heads).
template <typename T, bool VEC>
struct Sixteen {
    uint32_t w[VEC && sizeof(T) == 2 ? 8 : 16];

    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(T)); ++i) {
                const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p) + i);
                w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(static_cast<float>(p[i]));
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (VEC && sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};

// Two floats in one 64-bit register, and the packed operations on them.
struct Two {
    uint64_t v;
    __device__ __forceinline__ Two() {}
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void bits(uint32_t& a, uint32_t& b) const {
        asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(v));
    }
};
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(a.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return a;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(a.v) : "l"(a.v), "l"(b.v));
    return a;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(a.v) : "l"(a.v), "l"(b.v));
    return a;
}

// What turns a row's values into codes: codes8 computes rint(RN(RN(x - off) / s)), RN being the rounding to
// float32, from y, about 1 / s, without a division or a branch (51k tokens of 8 heads, bf16: 100 -> 63 us against
// divisions where a reciprocal came near a tie). It is Markstein's correction of a quotient by its exact remainder
// (kq_common.cuh names the paper), with an argument of its own for scales of 8 bits. q = RN(d y) is a few units u in the last place off d / s, and the scale has 8 bits, so
// q s and d are both whole multiples of u ulp(s): the remainder d - q s is one of a few hundred of them and exact. RN(q +
// (d - q s) y) then rounds a number within 2^-20 u of d / s; the nearest that d / s can be to the middle between two
// floats is 2^-9 u (d minus such a middle times s is such a multiple again, halved, and not 0: the
// product would need 25 bits), so it rounds to RN(d / s), ties of the codes included. x, off and s
// are multiplied by a power of two z that brings s between 2^-69 and 2^64, where nothing that can
// reach a code other than 0 is lost below the normal numbers.
struct Scaler {
    Two z, off, s, y;   // z, -off z, -s z, about 1 / (s z)
    __device__ __forceinline__ Scaler(float o, float step) {
        const float f = step < 0x1p-64f ? 0x1p64f : step > 0x1p64f ? 0x1p-64f : 1.0f, t = step * f;
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));   // within a unit in the last place
        z = Two(f, f), off = Two(-o * f, -o * f), s = Two(-t, -t), y = Two(r, r);
    }
};
// The codes of 8 values, the first in the lowest bits; of a row with scale 0, infinities or NaN, anything.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], const Scaler& g) {
    constexpr float kRound = 12582912.0f;   // 1.5 * 2^23: adding it rounds to a whole number, in the lowest bits
    uint32_t t[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const Two d = fma2(Two(x[j], x[j + 1]), g.z, g.off);
        const Two q = mul2(d, g.y);
        add2(fma2(fma2(q, g.s, d), g.y, q), Two(kRound, kRound)).bits(t[j], t[j + 1]);
    }
    const uint32_t even = __byte_perm(__byte_perm(t[0], t[2], 0x0040), __byte_perm(t[4], t[6], 0x0040), 0x5410);
    const uint32_t odd = __byte_perm(__byte_perm(t[1], t[3], 0x0040), __byte_perm(t[5], t[7], 0x0040), 0x5410);
    return even | odd << 4;
}

struct RowSource {
    const void* p[2];               // k, v
    int64_t token[2], head[2];      // strides in elements
};

constexpr int kRun = 8;     // consecutive tokens of a warp of append, one row of each at a time
constexpr int kBatch = 4;   // heads of a token that a warp of read takes at a time

// A token's place: its sequence, slot and the granule of head 0, or none.
struct Token {
    int b, t;            // sequence (-1: none), token in the granule
    int64_t slot;
    uint8_t* g;          // granule of head 0, or nullptr: no such slot or page
};
__device__ __forceinline__ Token locate(const KvView& c, int b, int64_t slot, int64_t most) {
    Token k = {b, 0, slot, nullptr};
    if (slot >= 0 && slot < most) {
        k.g = kv_granule(c, b, 0, slot);
        k.t = static_cast<int>(slot % kGranule);
    }
    return k;
}

template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kThreads, VEC && sizeof(T) == 2 ? 4 : 3) kv_append_kernel(KvView c, RowSource src, int64_t tokens, int groups, int per,
                                                             const int32_t* __restrict__ start,
                                                             const int32_t* __restrict__ lens, int32_t* lens_out,
                                                             float* __restrict__ acc, int32_t* __restrict__ pos, int64_t S,
                                                             const int32_t* __restrict__ seen, int32_t* seen_out, int* info) {
    constexpr int kChunks = D / 64;   // of 16 values, to each of a row's four lanes
    const int64_t cap = kv_capacity(c);
    if (blockIdx.x == 0) {
        for (int b = threadIdx.x; b < c.batch; b += kThreads) {
            const int64_t add = max(static_cast<int64_t>(0), static_cast<int64_t>(start[b + 1]) - start[b]);
            const int64_t n = kv_length(lens, b, cap, info);
            if (n + add > cap) record_error(info, -KQ_ERR_INVALID_ARG);
            if (lens_out) lens_out[b] = static_cast<int32_t>(min(n + add, cap));
            if (seen_out) seen_out[b] = static_cast<int32_t>((seen ? seen[b] : n) + add);
        }
        if (threadIdx.x == 0 && (start[0] != 0 || start[c.batch] != tokens)) record_error(info, -KQ_ERR_INVALID_ARG);
    }
    const int lane = threadIdx.x & 31, in_row = lane & 3;
    const int head_bytes = c.page * (D + 8);
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kThreads / 32), items = (tokens + kRun - 1) / kRun * groups;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); item < items; item += warps) {
        const int64_t turn = groups == 1 ? item : item / groups, i = turn * kRun + (lane >> 2);   // the lane's token
        const int u0 = static_cast<int>(item - turn * groups) * per, u1 = min(u0 + per, 2 * c.kv_heads);
        // lane in_row of a row takes its values 16 in_row + 64 u ..; the first rows are asked for before their place is known
        const int64_t in = min(i, tokens - 1);
        const T* const key = static_cast<const T*>(src.p[0]) + in * src.token[0] + in_row * 16;
        const T* const value = static_cast<const T*>(src.p[1]) + in * src.token[1] + in_row * 16;
        Sixteen<T, VEC> raw[kChunks];
        auto row_of = [&](int unit) { return unit & 1 ? value + (unit >> 1) * src.head[1] : key + (unit >> 1) * src.head[0]; };
#pragma unroll
        for (int u = 0; u < kChunks; ++u) raw[u].load(row_of(u0) + 64 * u);
        const int b = i < tokens ? kv_sequence_of(start, c.batch, i) : -1;
        Token k = {-1, 0, 0, nullptr};   // b < 0 is recorded by the first block
        int32_t at_pos = 0;
        if (b >= 0) {
            const int64_t n = kv_length(lens, b, cap, info), index = i - start[b];
            k = locate(c, b, n + index, cap);
            if (!k.g || ((acc || pos) && k.slot >= S)) record_error(info, -KQ_ERR_INVALID_ARG);
            if (pos) at_pos = static_cast<int32_t>((seen ? seen[b] : n) + index);
        }
        const bool there = k.g != nullptr;
        uint8_t* const codes0 = k.g + kv_code_at(D, 0, k.t) + in_row * 8;   // of head 0's key
        const int params0 = kv_param_at(D, 0, k.t) - kv_code_at(D, 0, k.t) - in_row * 8;
        const int64_t slot0 = static_cast<int64_t>(b) * c.kv_heads * S + k.slot;
        for (int unit = u0; unit < u1; ++unit) {   // all lanes go along; what has no place is not written
            const int which = unit & 1, h = unit >> 1;
            const T* const next = row_of(min(unit + 1, u1 - 1));
            uint8_t* const at = codes0 + h * static_cast<int64_t>(head_bytes);
            uint2* const codes = reinterpret_cast<uint2*>(at + which * kv_code_at(D, 1, 0));
            uint32_t* const params = reinterpret_cast<uint32_t*>(at + params0 + which * (kGranule * 4));
            // a NaN among the values stays in both
            float lo = raw[0].get(0), hi = lo;
#pragma unroll
            for (int u = 0; u < kChunks; ++u)
#pragma unroll
                for (int j = 0; j < 16; j += 2) {
                    const float x = raw[u].get(j), z = raw[u].get(j + 1);
                    asm("min.NaN.f32 %0, %0, %1, %2;" : "+f"(lo) : "f"(x), "f"(z));
                    asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(hi) : "f"(x), "f"(z));
                }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                const float l = __shfl_xor_sync(0xffffffffu, lo, o), t = __shfl_xor_sync(0xffffffffu, hi, o);
                asm("min.NaN.f32 %0, %0, %1;" : "+f"(lo) : "f"(l));
                asm("max.NaN.f32 %0, %0, %1;" : "+f"(hi) : "f"(t));
            }
            // down to bf16: negative values get a larger magnitude; up to bf16: the scale is >= 0
            const uint32_t lb = __float_as_uint(lo);
            const uint32_t ob = (lb + ((lb >> 31) ? 0xFFFFu : 0u)) & 0xFFFF0000u;
            const float off = __uint_as_float(ob);
            const uint32_t qb = __float_as_uint(__fdiv_rn(__fsub_rn(hi, off), 15.0f)), sb = (qb + 0xFFFFu) & 0xFFFF0000u;
            const float s = __uint_as_float(sb);
            const bool fine = qb <= 0x7F7F0000u, use = fine && sb;   // not NaN, not infinite, nor to become so
            const Scaler grid(off, s);
#pragma unroll
            for (int u = 0; u < kChunks; ++u) {
                uint32_t word[2];
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = raw[u].get(8 * v + j);
                    word[v] = use ? codes8(x, grid) : 0u;
                }
                if (there && KQ_IN_RANGE(reinterpret_cast<uint8_t*>(codes + 4 * u) - c.data, kv_pool_bytes(c) - 7))
                    codes[4 * u] = make_uint2(word[0], word[1]);
                if (unit + 1 < u1) raw[u].load(next + 64 * u);
            }
            if (there && in_row == 0) {
                if (KQ_IN_RANGE(reinterpret_cast<uint8_t*>(params) - c.data, kv_pool_bytes(c) - 3))
                    *params = fine ? (sb >> 16) | ob : 0x7FC07FC0u;
                const int64_t slot = slot0 + h * S;
                if (which == 0 && (acc || pos) && k.slot < S && KQ_IN_RANGE(slot, static_cast<int64_t>(c.batch) * c.kv_heads * S)) {
                    if (acc) acc[slot] = 0.0f;
                    if (pos) pos[slot] = at_pos;
                }
            }
        }
    }
}

// SHIFT: 1 << SHIFT tokens to a warp at a time, fewer heads of each. Otherwise few heads leave lanes
// idle: 51k tokens of one head in 11 instead of 20 us, of two in 18 instead of 23.
template <typename T, int D, int SHIFT>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(KvView c, int groups, int per, const int32_t* __restrict__ start,
                                                           const int32_t* __restrict__ first,
                                                           const int32_t* __restrict__ lens, int64_t tokens,
                                                           T* __restrict__ k_out, T* __restrict__ v_out, int* info) {
    constexpr int kLanes = D / 8, kRowsAtOnce = 32 / kLanes, kRounds = kBatch / (kRowsAtOnce / 2);
    const int lane = threadIdx.x & 31, in_row = lane % kLanes, sub = lane / kLanes, which = sub & 1;
    const int64_t cap = kv_capacity(c);
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
    constexpr int kSide = kBatch >> SHIFT;   // heads of a token at a time
    const int64_t items = ((tokens + (1 << SHIFT) - 1) >> SHIFT) * groups;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); item < items; item += warps) {
        const int64_t turn = groups == 1 ? item : item / groups, i0 = turn << SHIFT;
        const int h0 = static_cast<int>(item - turn * groups) * per, h1 = min(h0 + per, c.kv_heads);
        // a lane looks up one of the tokens
        const int64_t i = SHIFT ? i0 + (lane & ((1 << SHIFT) - 1)) : i0;
        int b = -1;
        if (SHIFT == 0) b = kv_sequence_of_warp(start, c.batch, i);
        else if (i < tokens) b = kv_sequence_of(start, c.batch, i);
        Token k = {-1, 0, 0, nullptr};
        if (b >= 0) {
            const int64_t n = lens ? kv_length(lens, b, cap, info) : cap;
            k = locate(c, b, (first ? first[b] : 0) + (i - start[b]), n);
            if (k.slot < 0 || (k.slot < n && !k.g)) record_error(info, -KQ_ERR_INVALID_ARG);
        }
        T* out = (which ? v_out : k_out) + i0 * c.kv_heads * D + in_row * 8;
        for (int hb = h0; hb < h1; hb += kSide) {
            uint32_t word[kRounds], prm[kRounds];
#pragma unroll
            for (int u = 0; u < kRounds; ++u) {
                const int at = u * (kRowsAtOnce / 2) + (sub >> 1), of = at >> (2 - SHIFT), h = hb + (SHIFT ? at & (kSide - 1) : at);
                const uint8_t* g = k.g;
                int t = k.t;
                if (SHIFT) {
                    g = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(k.g), of));
                    t = __shfl_sync(0xffffffffu, k.t, of);
                }
                word[u] = prm[u] = 0;
                if (g && h < h1) {
                    g += h * kv_head_bytes(c);
                    word[u] = reinterpret_cast<const uint32_t*>(g + kv_code_at(D, which, t))[in_row];
                    prm[u] = *reinterpret_cast<const uint32_t*>(g + kv_param_at(D, which, t));
                }
            }
#pragma unroll
            for (int u = 0; u < kRounds; ++u) {
                const int at = u * (kRowsAtOnce / 2) + (sub >> 1), h = hb + (SHIFT ? at & (kSide - 1) : at);
                const int of = at >> (2 - SHIFT);
                if (h >= h1 || (SHIFT && i0 + of >= tokens)) continue;
                const float s = kv_scale(prm[u]), off = kv_offset(prm[u]);   // 0 where there is nothing to read
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = fmaf(s, static_cast<float>((word[u] >> (4 * j)) & 15u), off);
                T* dst = out + static_cast<int64_t>(SHIFT ? of * c.kv_heads + h : h) * D;
                if (!KQ_IN_RANGE(dst - (which ? v_out : k_out), tokens * c.kv_heads * D - 7)) continue;
                if constexpr (sizeof(T) == 2) {
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
                        w[j] = *reinterpret_cast<const uint32_t*>(&p);
                    }
                    *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                } else {   // streamed past L2: 105 -> 95 us for 51k tokens of 8 heads; bf16 rows lose by it (114 -> 125 us)
                    __stcs(reinterpret_cast<float4*>(dst), make_float4(x[0], x[1], x[2], x[3]));
                    __stcs(reinterpret_cast<float4*>(dst) + 1, make_float4(x[4], x[5], x[6], x[7]));
                }
            }
        }
    }
}

// Heads to a warp: all of a token's, unless that leaves SMs without work.
struct Cut {
    int groups, per;
    unsigned grid;
};
Cut cut(int64_t tokens, int kv_heads) {
    Cut k;
    const int64_t want = cdiv(static_cast<int64_t>(num_sms()) * 16, std::max<int64_t>(1, tokens));
    const int64_t most = cdiv(kv_heads, kBatch);
    k.groups = static_cast<int>(std::max<int64_t>(1, std::min(want, most)));
    k.per = static_cast<int>(cdiv(cdiv(kv_heads, k.groups), kBatch) * kBatch);
    k.groups = static_cast<int>(cdiv(kv_heads, k.per));
    k.grid = static_cast<unsigned>(std::max<int64_t>(
        1, std::min<int64_t>(cdiv(tokens * k.groups, kThreads / 32), static_cast<int64_t>(num_sms()) * 16)));
    return k;
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
    // the first block writes its outputs while the others read these
    auto read_too = [&](const int32_t* out) {
        return kv_overlap(out, c.batch, start, c.batch + 1) || kv_overlap(out, c.batch, lens, c.batch) ||
               kv_overlap(out, c.batch, seen, c.batch);
    };
    if (T < 0 || T > 0x7fffffffll || !start || !lens || (T > 0 && (!k || !v)) || ((acc || pos) && S < 1) ||
        read_too(lens_out) || read_too(seen_out) || kv_overlap(lens_out, c.batch, seen_out, c.batch) ||
        ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & (es - 1))) {
        set_error("kq_kv_append: start, lens, k, v must not be NULL, 0 <= T < 2^31, S >= 1 with acc or pos, lens_out and "
                  "seen_out apart from each other and from start, lens and seen");
        return KQ_ERR_INVALID_ARG;
    }
    RowSource src = {{k, v}, {k_token_stride, v_token_stride}, {k_head_stride, v_head_stride}};
    bool vec = true;
    for (int w = 0; w < 2; ++w)
        vec = vec && !(reinterpret_cast<uintptr_t>(src.p[w]) & 15u) && !((src.token[w] * es) & 15u) && !((src.head[w] * es) & 15u);
    // four units (a key or value row of each token) to a warp, unless that leaves SMs without work: for 51k tokens of 8
    // heads, fp32, 81 us (one: 95, two: 83, eight: 84, sixteen: 85)
    const int64_t runs = cdiv(T, kRun), units = 2 * c.kv_heads;
    const int per = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(4, runs * units / (num_sms() * 64))));
    const int groups = static_cast<int>(cdiv(units, per));
    const unsigned grid = static_cast<unsigned>(std::max<int64_t>(
        1, std::min<int64_t>(cdiv(runs * groups, kThreads / 32), static_cast<int64_t>(num_sms()) * 16)));
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
#define KQ_APPEND(TY, DIM, VEC)                                                                                            \
    kv_append_kernel<TY, DIM, VEC><<<grid, kThreads, 0, stream>>>(c, src, T, groups, per, start, lens, lens_out, acc, pos, S, \
                                                                  seen, seen_out, info)
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
    const int shift = c.kv_heads == 1 ? 2 : c.kv_heads == 2 ? 1 : 0;
    const Cut by = cut((T + (1 << shift) - 1) >> shift, c.kv_heads);
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
#define KQ_READ_BY(TY, DIM, SHIFT)                                                                                             \
    kv_read_kernel<TY, DIM, SHIFT><<<by.grid, kThreads, 0, stream>>>(c, by.groups, by.per, start, first, lens, T, \
                                                                     static_cast<TY*>(k), static_cast<TY*>(v), info)
#define KQ_READ(TY, DIM) shift == 0 ? KQ_READ_BY(TY, DIM, 0) : shift == 1 ? KQ_READ_BY(TY, DIM, 1) : KQ_READ_BY(TY, DIM, 2)
    if (dtype == KQ_BF16) {
        if (c.dim == 128) KQ_READ(__nv_bfloat16, 128);
        else KQ_READ(__nv_bfloat16, 64);
    } else {
        if (c.dim == 128) KQ_READ(float, 128);
        else KQ_READ(float, 64);
    }
#undef KQ_READ_BY
#undef KQ_READ
    KQ_LAUNCH_CHECK("kv_read_kernel");
    return KQ_OK;
}
