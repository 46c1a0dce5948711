// kq_qk_rotate and kq_qk_rotate_grad: norm and rotary positions of queries and keys, one pass over the rows.
//
// Mathematics. A row x of D values (one token, one head), normed where a weight w is given:
//     n = x r w,  r = (mean(x^2) + eps)^(-1/2),
// then the first R dimensions are rotated in pairs (a, b), dimensions (j, j + R / 2) or (2 j, 2 j + 1), by the angle
// of the token's position and pair j:  (a', b') = s (a cos - b sin, b cos + a sin); the others stay as they are.
// Backwards: g = the transposed rotation of gy; with u = g w and h = x r,
//     gx = r (u - h mean(u h)),  gw = sum over rows of g h.
// Frequencies are 64-bit fractions of a turn for one position: the whole-number product with a position wraps at a
// turn, so the angle of position 2^31 is as exact as that of position 1. Of the product's fraction of a turn the
// upper 32 bits are used (1.5e-9 rad), rounded to fp32 (within 2^-25 of a turn): 2e-7 of the row's size.
//
// What bounds it: bytes, 2 elements moved for each forward, 3 backward, against about 10 instructions an
// element. So: 16 bytes to a lane, G lanes to a row, cos and sin computed once a token (a table in shared memory, from
// which each lane takes its own into registers for all the heads it goes through), partners exchanged by
// shuffles, and kAhead rows of loads in flight to a lane.
#include <algorithm>
#include <atomic>

#include "kv_common.cuh"
#include "pdl.cuh"

namespace kq {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;          // rows of a lane in flight
constexpr int kMaxDim = 256;
constexpr int kPairs = 0, kHalves = 1, kHalvesOdd = 2;   // layouts; odd: R / 2 is no multiple of a vector

template <typename T>
struct Rows {
    const T* x;
    const T* gy;       // backward
    T* out;
    const T* w;        // nullptr: no norm
    int64_t x_token, x_head, g_token, g_head, o_token, o_head;   // strides in elements
    int32_t heads;
};
template <typename T>
struct Rotate {
    Rows<T> s[2];      // queries, keys
    int64_t tokens;
    const uint64_t* freq;
    const int32_t *pos, *start, *first;
    int32_t batch, dim, half;        // half: pairs
    int32_t per;       // tokens of a block at a time, a power of two
    int32_t part;      // heads of a block
    float scale, eps;
    bool vec;          // every row can be moved 16 bytes at a time
    float* sums;       // backward: [blocks][2][dim] of weight gradients, or nullptr
};

template <typename T>
struct Lane {
    static constexpr int E = 16 / sizeof(T);
    static __device__ __forceinline__ uint4 load(const T* p, bool vec, int n) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (vec) {
            if (n > 0) u = *reinterpret_cast<const uint4*>(p);
        } else {
            T* e = reinterpret_cast<T*>(&u);
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i < n) e[i] = p[i];
        }
        return u;
    }
    static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[E]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < E; ++i)
            x[i] = __uint_as_float(sizeof(T) == 4 ? w[i % 4] : i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    static __device__ __forceinline__ void store(T* p, bool vec, int n, const float (&x)[E]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = __float_as_uint(x[i]);
            } else {
                const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&t);
            }
        }
        uint4 u = make_uint4(w[0], w[1], w[2], w[3]);
        if (vec) {
            if (n > 0) *reinterpret_cast<uint4*>(p) = u;
        } else {
            const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i < n) p[i] = e[i];
        }
    }
};

template <int G>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A lane's share of a row, NV vectors l, l + G, ..: cos and sin (of the sign that the partner enters with) of its dimensions.
template <typename T, int G, int NV, int MODE>
struct Share {
    static constexpr int E = Lane<T>::E;
    float c[NV][E], s[NV][E];
    int n[NV], turned[NV];     // dimensions of a vector, and how many of them are rotated
    int l;

    __device__ __forceinline__ Share(int l_, int dim) : l(l_) {
#pragma unroll
        for (int k = 0; k < NV; ++k) n[k] = min(E, max(0, dim - (l + k * G) * E));
    }
    __device__ __forceinline__ int dim_of(int k, int e) const { return (l + k * G) * E + e; }
    __device__ __forceinline__ void take(const float2* table, int half) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            turned[k] = min(E, max(0, 2 * half - (l + k * G) * E));
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = dim_of(k, e);
                const bool in = e < turned[k], second = MODE == kPairs ? e & 1 : i >= half;
                const float2 t = table[in ? (MODE == kPairs ? i / 2 : second ? i - half : i) : 0];
                c[k][e] = t.x;
                s[k][e] = second ? t.y : -t.y;
            }
        }
    }
    // y = rotated x; BACK: by the transposed matrix. xch: D floats of the row in shared memory (odd halves). Whole warps call it.
    template <bool BACK>
    __device__ __forceinline__ void turn(float (&x)[NV][E], int half, float* xch) const {
        float y[NV][E];   // partners
        if constexpr (MODE == kPairs) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) y[k][e] = x[k][e ^ 1];
        } else if constexpr (MODE == kHalves) {
            const int step = half / E;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int v = l + k * G, from = v < step ? v + step : v - step;   // past R: not used
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float got = __shfl_sync(0xffffffffu, x[0][e], from, G);
                    if constexpr (NV == 2) {
                        const float other = __shfl_sync(0xffffffffu, x[1][e], from, G);
                        if (from >= G) got = other;
                    }
                    y[k][e] = got;
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e < n[k]) xch[dim_of(k, e)] = x[k][e];
            __syncwarp();
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int i = dim_of(k, e);
                    y[k][e] = e < turned[k] ? xch[i < half ? i + half : i - half] : 0.0f;
                }
            __syncwarp();
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < turned[k]) x[k][e] = fmaf(BACK ? -s[k][e] : s[k][e], y[k][e], c[k][e] * x[k][e]);
    }
};

// cos and sin of the block's tokens from t0 on; whether a token has a position.
template <typename T>
__device__ __forceinline__ void fill_table(const Rotate<T>& p, int64_t t0, float2* table, int* known) {
    for (int i = threadIdx.x; i < p.per * max(1, p.half); i += kThreads) {
        const int a = i / max(1, p.half), j = i - a * max(1, p.half);
        const int64_t t = t0 + a;
        int64_t pos = t;
        bool is = t < p.tokens;
        if (is && p.pos) {
            pos = p.pos[t];
        } else if (is && p.start) {
            const int b = kv_sequence_of(p.start, p.batch, t);
            is = b >= 0;
            if (is) pos = p.first[b] + (t - p.start[b]);
        }
        if (j == 0) known[a] = is;
        if (j < p.half) {
            const int32_t turn = static_cast<int32_t>((static_cast<uint64_t>(pos) * p.freq[j]) >> 32);
            float s, c;
            sincospif(static_cast<float>(turn) * 0x1p-31f, &s, &c);
            table[i] = make_float2(c * p.scale, s * p.scale);
        }
    }
}

// Blocks (tokens, heads): `per` tokens, the slots of G lanes dealt to them in turn, each going through heads.
template <typename T, int G, int NV, int MODE>
__global__ void __launch_bounds__(kThreads) qk_rotate_kernel(const Rotate<T> p) {
    constexpr int E = Lane<T>::E, kSlots = kThreads / G;
    extern __shared__ __align__(16) uint8_t smem[];
    float2* table = reinterpret_cast<float2*>(smem);
    __shared__ int known[kSlots];
    const int slot = threadIdx.x / G, mine = slot & (p.per - 1);
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.per, t = t0 + mine;
    float* xch = reinterpret_cast<float*>(table + p.per * max(1, p.half)) + slot * (MODE == kHalvesOdd ? p.dim : 0);
    Share<T, G, NV, MODE> sh(threadIdx.x % G, p.dim);
    const int heads = min(p.s[0].heads + p.s[1].heads - static_cast<int>(blockIdx.y) * p.part, p.part);
    const int h0 = blockIdx.y * p.part, step = kSlots / p.per, turns = (heads + step - 1) / step;
    pdl_wait();
    pdl_launch_dependents();
    uint4 raw[kAhead][NV], w[2][NV];
    bool is = t < p.tokens;
    const bool any = p.s[0].w || p.s[1].w;
    auto head_of = [&](int i) { return slot / p.per + i * step; };   // among the block's heads
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int hh = head_of(i0 + u), h = h0 + hh, side = h >= p.s[0].heads;
            const Rows<T>& s = p.s[side];
            const T* src = s.x + t * s.x_token + static_cast<int64_t>(side ? h - p.s[0].heads : h) * s.x_head;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (is && hh < heads) raw[u][k] = Lane<T>::load(src + sh.dim_of(k, 0), p.vec, sh.n[k]);
        }
    };
    fetch(0);
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int k = 0; k < NV; ++k)
            w[side][k] = p.s[side].w ? Lane<T>::load(p.s[side].w + sh.dim_of(k, 0), p.vec, sh.n[k]) : make_uint4(0, 0, 0, 0);
    fill_table(p, t0, table, known);
    __syncthreads();
    sh.take(table + mine * p.half, p.half);
    is = is && known[mine];
    for (int i0 = 0; i0 < turns; i0 += kAhead) {
        if (i0 > 0) fetch(i0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i0 + u >= turns) break;
            const int hh = head_of(i0 + u), h = h0 + hh, side = h >= p.s[0].heads;
            const Rows<T>& s = p.s[side];
            const bool here = is && hh < heads;
            float x[NV][E];
#pragma unroll
            for (int k = 0; k < NV; ++k) Lane<T>::unpack(here ? raw[u][k] : make_uint4(0, 0, 0, 0), x[k]);
            float sum = 0.0f;
            if (any) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e) sum = fmaf(x[k][e], x[k][e], sum);
                sum = row_sum<G>(sum);
            }
            if (s.w) {
                const float r = __frsqrt_rn(sum / static_cast<float>(p.dim) + p.eps);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    float g[E];
                    Lane<T>::unpack(side ? w[1][k] : w[0][k], g);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[k][e] = x[k][e] * r * g[e];
                }
            }
            sh.template turn<false>(x, p.half, xch);
            if (here) {
                T* dst = s.out + t * s.o_token + static_cast<int64_t>(side ? h - p.s[0].heads : h) * s.o_head;
#pragma unroll
                for (int k = 0; k < NV; ++k) Lane<T>::store(dst + sh.dim_of(k, 0), p.vec, sh.n[k], x[k]);
            }
        }
    }
}

// The same backwards. Blocks stay and go through the tokens, so that the weights' gradients are summed in registers, then over
// the block's slots in order, then (rotate_sums_kernel) over the blocks in order.
template <typename T, int G, int NV, int MODE>
__global__ void __launch_bounds__(kThreads) qk_rotate_grad_kernel(const Rotate<T> p) {
    constexpr int E = Lane<T>::E, kSlots = kThreads / G;
    extern __shared__ __align__(16) uint8_t smem[];
    float2* table = reinterpret_cast<float2*>(smem);
    __shared__ int known[kSlots];
    const int slot = threadIdx.x / G, mine = slot & (p.per - 1);
    float* xch = reinterpret_cast<float*>(table + p.per * max(1, p.half)) + slot * (MODE == kHalvesOdd ? p.dim : 0);
    Share<T, G, NV, MODE> sh(threadIdx.x % G, p.dim);
    const int heads = p.s[0].heads + p.s[1].heads, step = kSlots / p.per;
    pdl_wait();
    pdl_launch_dependents();
    uint4 w[2][NV];
    float gw[2][NV][E];
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            w[side][k] = p.s[side].w ? Lane<T>::load(p.s[side].w + sh.dim_of(k, 0), p.vec, sh.n[k]) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < E; ++e) gw[side][k][e] = 0.0f;
        }
    const float over = 1.0f / static_cast<float>(p.dim);
    for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * p.per; t0 < p.tokens; t0 += static_cast<int64_t>(gridDim.x) * p.per) {
        const int64_t t = t0 + mine;
        __syncthreads();
        fill_table(p, t0, table, known);
        __syncthreads();
        sh.take(table + mine * p.half, p.half);
        const bool is = known[mine];
        // queries, then keys, so that each side's sums stay where they are
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const Rows<T>& s = p.s[side];
            const bool norm = s.w != nullptr;
            for (int i0 = 0; i0 * step < s.heads; i0 += kAhead / 2) {
                uint4 rx[kAhead / 2][NV], rg[kAhead / 2][NV];
#pragma unroll
                for (int u = 0; u < kAhead / 2; ++u) {
                    const int h = slot / p.per + (i0 + u) * step;
                    const bool here = is && h < s.heads;
                    const T* gy = s.gy + t * s.g_token + static_cast<int64_t>(h) * s.g_head;
                    const T* x = s.x + t * s.x_token + static_cast<int64_t>(h) * s.x_head;
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        rg[u][k] = rx[u][k] = make_uint4(0, 0, 0, 0);
                        if (here) rg[u][k] = Lane<T>::load(gy + sh.dim_of(k, 0), p.vec, sh.n[k]);
                        if (here && norm) rx[u][k] = Lane<T>::load(x + sh.dim_of(k, 0), p.vec, sh.n[k]);
                    }
                }
#pragma unroll
                for (int u = 0; u < kAhead / 2; ++u) {
                    if ((i0 + u) * step >= s.heads) break;
                    const int h = slot / p.per + (i0 + u) * step;
                    float g[NV][E], x[NV][E];
#pragma unroll
                    for (int k = 0; k < NV; ++k) {
                        Lane<T>::unpack(rg[u][k], g[k]);
                        Lane<T>::unpack(rx[u][k], x[k]);
                    }
                    sh.template turn<true>(g, p.half, xch);
                    if (norm) {
                        float sum = 0.0f, dot = 0.0f;
#pragma unroll
                        for (int k = 0; k < NV; ++k) {
                            float y[E];
                            Lane<T>::unpack(w[side][k], y);
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                sum = fmaf(x[k][e], x[k][e], sum);
                                dot = fmaf(g[k][e] * y[e], x[k][e], dot);
                            }
                        }
                        sum = row_sum<G>(sum);
                        dot = row_sum<G>(dot);
                        const float r = __frsqrt_rn(sum * over + p.eps), f = dot * over * r * r;
#pragma unroll
                        for (int k = 0; k < NV; ++k) {
                            float y[E];
                            Lane<T>::unpack(w[side][k], y);
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                gw[side][k][e] = fmaf(g[k][e], x[k][e] * r, gw[side][k][e]);
                                g[k][e] = r * fmaf(-f, x[k][e], g[k][e] * y[e]);
                            }
                        }
                    }
                    if (is && h < s.heads) {
                        T* dst = s.out + t * s.o_token + static_cast<int64_t>(h) * s.o_head;
#pragma unroll
                        for (int k = 0; k < NV; ++k) Lane<T>::store(dst + sh.dim_of(k, 0), p.vec, sh.n[k], g[k]);
                    }
                }
            }
        }
    }
    if (!p.sums) return;
    // slots in order, one vector of a lane at a time
    float* all = reinterpret_cast<float*>(smem);   // [kSlots][dim]
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < sh.n[k]) all[slot * p.dim + sh.dim_of(k, e)] = gw[side][k][e];
        __syncthreads();
        for (int i = threadIdx.x; i < p.dim; i += kThreads) {
            float sum = 0.0f;
            for (int q = 0; q < kSlots; ++q) sum += all[q * p.dim + i];
            p.sums[(static_cast<int64_t>(blockIdx.x) * 2 + side) * p.dim + i] = sum;
        }
    }
}

// gw = the blocks' sums: block (32 dimensions, side), warps share the blocks' rows.
__global__ void __launch_bounds__(1024) rotate_sums_kernel(const float* __restrict__ sums, int blocks, int dim, float* gq, float* gk) {
    __shared__ float part[32][33];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane, side = blockIdx.y;
    float* out = side ? gk : gq;
    float s = 0.0f;
    if (i < dim)
        for (int b = warp; b < blocks; b += 32) s += sums[(static_cast<int64_t>(b) * 2 + side) * dim + i];
    part[warp][lane] = s;
    __syncthreads();
    if (warp > 0 || i >= dim || !out) return;
    s = 0.0f;
    for (int q = 0; q < 32; ++q) s += part[q][lane];
    out[i] = s;
}

constexpr int kMaxBlocks = 512;   // that a workspace has room for the sums of
int64_t grad_blocks(int64_t tokens) { return std::min<int64_t>(tokens, kMaxBlocks); }

template <typename T, int G, int NV, int MODE>
kq_status launch(Rotate<T>& p, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    constexpr int kSlots = kThreads / G;
    const int heads = p.s[0].heads + p.s[1].heads;
    const int64_t sms = num_sms();
    // several tokens to a block where there are many, so that the table costs little; the heads over several blocks
    // where there are few
    p.per = 1;
    while (p.per < kSlots && p.per < 4 && p.tokens >= 2 * p.per * sms * 4) p.per *= 2;
    p.part = heads;
    if (p.tokens < 2 * sms) p.part = static_cast<int>(std::max<int64_t>(std::min(heads, kSlots), cdiv(heads, std::max<int64_t>(1, 2 * sms / p.tokens))));
    size_t smem = p.per * std::max(1, p.half) * sizeof(float2) + (MODE == kHalvesOdd ? kSlots * p.dim * sizeof(float) : 0);
    if (!back) {
        const dim3 grid(static_cast<unsigned>(cdiv(p.tokens, p.per)), static_cast<unsigned>(cdiv(heads, p.part)));
        KQ_CUDA(launch_after(qk_rotate_kernel<T, G, NV, MODE>, grid, dim3(kThreads), smem, stream, p));
        count_launch();
        return KQ_OK;
    }
    const int blocks = static_cast<int>(std::min({grad_blocks(p.tokens), cdiv(p.tokens, p.per), sms * 3}));
    if (p.sums) smem = std::max(smem, kSlots * p.dim * sizeof(float));
    KQ_CUDA(launch_after(qk_rotate_grad_kernel<T, G, NV, MODE>, dim3(blocks), dim3(kThreads), smem, stream, p));
    count_launch();
    if (p.sums) {
        KQ_CUDA(launch_after(rotate_sums_kernel, dim3(static_cast<unsigned>(cdiv(p.dim, 32)), 2), dim3(1024), 0, stream,
                             static_cast<const float*>(p.sums), blocks, static_cast<int>(p.dim), gqw, gkw));
        count_launch();
    }
    return KQ_OK;
}

template <typename T, int G, int NV>
kq_status launch_mode(Rotate<T>& p, bool pairs, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    if (pairs) return launch<T, G, NV, kPairs>(p, back, gqw, gkw, stream);
    if (p.half % Lane<T>::E == 0) return launch<T, G, NV, kHalves>(p, back, gqw, gkw, stream);
    return launch<T, G, NV, kHalvesOdd>(p, back, gqw, gkw, stream);
}
kq_status launch_dim(Rotate<__nv_bfloat16>& p, bool pairs, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    if (p.dim <= 64) return launch_mode<__nv_bfloat16, 8, 1>(p, pairs, back, gqw, gkw, stream);
    if (p.dim <= 128) return launch_mode<__nv_bfloat16, 16, 1>(p, pairs, back, gqw, gkw, stream);
    return launch_mode<__nv_bfloat16, 32, 1>(p, pairs, back, gqw, gkw, stream);
}
kq_status launch_dim(Rotate<float>& p, bool pairs, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    if (p.dim <= 64) return launch_mode<float, 16, 1>(p, pairs, back, gqw, gkw, stream);
    if (p.dim <= 128) return launch_mode<float, 32, 1>(p, pairs, back, gqw, gkw, stream);
    return launch_mode<float, 32, 2>(p, pairs, back, gqw, gkw, stream);
}

// What both calls check of a set of rows.
kq_status check_rows(const char* who, const char* name, const kq_heads* h, size_t es) {
    if (!h || !h->data || h->heads < 1 || (reinterpret_cast<uintptr_t>(h->data) & (es - 1))) {
        set_error("%s: %s needs data aligned to its type and at least one head", who, name);
        return KQ_ERR_INVALID_ARG;
    }
    return KQ_OK;
}

template <typename T>
kq_status run(const kq_rotation* r, int64_t tokens, int64_t dim, const kq_heads* q, const kq_heads* k,
              const kq_heads* gq, const kq_heads* gk, const kq_heads* qo, const kq_heads* ko, const void* qw, const void* kw,
              float eps, float* gqw, float* gkw, float* sums, cudaStream_t stream) {
    Rotate<T> p = {};
    const kq_heads* in[2] = {q, k};
    const kq_heads* g[2] = {gq, gk};
    const kq_heads* out[2] = {qo, ko};
    const void* w[2] = {qw, kw};
    uintptr_t bits = 0;   // whatever is not a multiple of 16 bytes
    for (int i = 0; i < 2; ++i) {
        Rows<T>& s = p.s[i];
        if (!out[i]) continue;   // no keys
        s.heads = static_cast<int32_t>(out[i]->heads);
        s.out = static_cast<T*>(out[i]->data);
        s.o_token = out[i]->token_stride, s.o_head = out[i]->head_stride;
        s.w = static_cast<const T*>(w[i]);
        bits |= reinterpret_cast<uintptr_t>(s.out) | reinterpret_cast<uintptr_t>(s.w) | (s.o_token | s.o_head) * sizeof(T);
        if (in[i]) {
            s.x = static_cast<const T*>(in[i]->data);
            s.x_token = in[i]->token_stride, s.x_head = in[i]->head_stride;
            bits |= reinterpret_cast<uintptr_t>(s.x) | (s.x_token | s.x_head) * sizeof(T);
        }
        if (g[i]) {
            s.gy = static_cast<const T*>(g[i]->data);
            s.g_token = g[i]->token_stride, s.g_head = g[i]->head_stride;
            bits |= reinterpret_cast<uintptr_t>(s.gy) | (s.g_token | s.g_head) * sizeof(T);
        }
    }
    p.tokens = tokens;
    p.freq = reinterpret_cast<const uint64_t*>(r->freq);
    p.pos = r->pos, p.start = r->start, p.first = r->first;
    p.batch = static_cast<int32_t>(r->batch);
    p.dim = static_cast<int32_t>(dim);
    p.half = static_cast<int32_t>(r->rot / 2);
    p.scale = r->scale;
    p.eps = eps;
    p.vec = !((bits | dim * sizeof(T)) & 15u);
    p.sums = sums;
    return launch_dim(p, r->interleaved != 0, gq != nullptr, gqw, gkw, stream);
}

// The arguments that both calls share. side i needs inputs where it has outputs.
kq_status check(const char* who, const kq_rotation* r, int dtype, int64_t T, int64_t dim, const kq_heads* const (&in)[2],
                const kq_heads* const (&out)[2], const void* const (&w)[2], float eps) {
    if (dtype != KQ_BF16 && dtype != KQ_F32) {
        set_error("%s: dtype must be KQ_BF16 or KQ_F32", who);
        return KQ_ERR_UNSUPPORTED;
    }
    if (dim > kMaxDim) {
        set_error("%s: dim must be at most %d", who, kMaxDim);
        return KQ_ERR_UNSUPPORTED;
    }
    const size_t es = dtype == KQ_BF16 ? 2 : 4;
    if (T < 0 || T > 0x7fffffffll || dim < 1 || !r || r->rot < 0 || r->rot > dim || (r->rot & 1) || (r->rot > 0 && !r->freq) ||
        !(r->scale - r->scale == 0.0f) || (!r->start != !r->first) || (r->pos && r->start) ||
        (r->start && (r->batch < 1 || r->batch > 0x7fffffffll)) || (reinterpret_cast<uintptr_t>(r->freq) & 7u)) {
        set_error("%s: 0 <= T < 2^31, an even rot up to dim with its frequencies, a finite scale, and positions from pos, from "
                  "start and first together, or from neither, needed", who);
        return KQ_ERR_INVALID_ARG;
    }
    if (!out[0] || !in[0] || (!in[1]) != (!out[1])) {
        set_error("%s: queries are needed, and keys with an output of their own or neither", who);
        return KQ_ERR_INVALID_ARG;
    }
    for (int i = 0; i < 2; ++i) {
        if (!out[i]) continue;
        if (T > 0) {
            KQ_TRY(check_rows(who, i ? "k_out" : "q_out", out[i], es));
            KQ_TRY(check_rows(who, i ? "k" : "q", in[i], es));
        }
        if (in[i]->heads != out[i]->heads || out[i]->heads < 1 || out[i]->heads > 65535) {
            set_error("%s: inputs and outputs must have the same heads, at most 65535", who);
            return KQ_ERR_INVALID_ARG;
        }
        if (w[i] && (!(eps >= 0.0f) || !(eps - eps == 0.0f) || (reinterpret_cast<uintptr_t>(w[i]) & (es - 1)))) {
            set_error("%s: norms need eps >= 0 and weights aligned to their type", who);
            return KQ_ERR_INVALID_ARG;
        }
    }
    return KQ_OK;
}

}  // namespace

KQ_DEBUG_UNIT(rotate)
}  // namespace kq

using namespace kq;

extern "C" kq_status kq_qk_rotate(const kq_rotation* r, int dtype, int64_t T, int64_t dim, const kq_heads* q, const kq_heads* k,
                                  const kq_heads* q_out, const kq_heads* k_out, const void* q_weight, const void* k_weight,
                                  float eps, kq_stream_t stream_) {
    KQ_TRY(check("kq_qk_rotate", r, dtype, T, dim, {q, k}, {q_out, k_out}, {q_weight, k_weight}, eps));
    if (T == 0) return KQ_OK;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (dtype == KQ_BF16)
        return run<__nv_bfloat16>(r, T, dim, q, k, nullptr, nullptr, q_out, k_out, q_weight, k_weight, eps, nullptr,
                                  nullptr, nullptr, stream);
    return run<float>(r, T, dim, q, k, nullptr, nullptr, q_out, k_out, q_weight, k_weight, eps, nullptr, nullptr,
                      nullptr, stream);
}

extern "C" size_t kq_qk_rotate_grad_workspace(int64_t T, int64_t dim) {
    if (T < 1 || dim < 1) return 0;
    return static_cast<size_t>(grad_blocks(T)) * 2 * dim * sizeof(float);
}

extern "C" kq_status kq_qk_rotate_grad(const kq_rotation* r, int dtype, int64_t T, int64_t dim, const kq_heads* q,
                                       const kq_heads* k, const kq_heads* gq, const kq_heads* gk, const kq_heads* q_out,
                                       const kq_heads* k_out, const void* q_weight, const void* k_weight, float eps,
                                       float* gq_weight, float* gk_weight, void* ws, size_t ws_bytes, kq_stream_t stream_) {
    const char* who = "kq_qk_rotate_grad";
    KQ_TRY(check(who, r, dtype, T, dim, {gq, gk}, {q_out, k_out}, {q_weight, k_weight}, eps));
    const kq_heads* in[2] = {q, k};
    const kq_heads* out[2] = {q_out, k_out};
    const void* w[2] = {q_weight, k_weight};
    const float* gw[2] = {gq_weight, gk_weight};
    for (int i = 0; i < 2; ++i) {
        if (gw[i] && (!w[i] || !out[i])) {
            set_error("%s: a weight's gradient needs the weight", who);
            return KQ_ERR_INVALID_ARG;
        }
        if (!out[i] || !w[i] || T == 0) continue;
        KQ_TRY(check_rows(who, i ? "k" : "q", in[i], dtype == KQ_BF16 ? 2 : 4));
        if (in[i]->heads != out[i]->heads) {
            set_error("%s: inputs and outputs must have the same heads", who);
            return KQ_ERR_INVALID_ARG;
        }
    }
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (T == 0) {
        for (float* g : {gq_weight, gk_weight})
            if (g) KQ_CUDA(cudaMemsetAsync(g, 0, dim * sizeof(float), stream));
        return KQ_OK;
    }
    const bool sums = gq_weight || gk_weight;
    if (sums && (!ws || ws_bytes < kq_qk_rotate_grad_workspace(T, dim) || (reinterpret_cast<uintptr_t>(ws) & 255u))) {
        set_error("%s: workspace must be 256-byte aligned and hold %zu bytes", who, kq_qk_rotate_grad_workspace(T, dim));
        return KQ_ERR_WORKSPACE;
    }
    float* s = sums ? static_cast<float*>(ws) : nullptr;
    if (dtype == KQ_BF16)
        return run<__nv_bfloat16>(r, T, dim, q, k, gq, gk, q_out, k_out, q_weight, k_weight, eps, gq_weight, gk_weight, s,
                                  stream);
    return run<float>(r, T, dim, q, k, gq, gk, q_out, k_out, q_weight, k_weight, eps, gq_weight, gk_weight, s, stream);
}
