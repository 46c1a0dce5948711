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
// What bounds it: bytes, 2 elements moved for each forward, 3 backward, against about 12 instructions an
// element. So a warp takes a token, or one for each of its groups of G lanes, by itself: it has the next two looks' loads in flight
// while it works on two (16 bytes to a lane, G lanes to a row, 32 / G rows a look), computes cos and sin of the tokens' pairs
// once, and exchanges partners by shuffles. Backwards the warps stay and go from token to token, the weights' sums in registers.
// Measured: 32768 tokens of 40 bf16 rows of 128, with norms, 120 us (5.6 TB/s, about 140 instructions for two rows of a
// warp); backwards 16384 tokens 106 us (4.8 TB/s, 215 instructions).
#include <algorithm>
#include <atomic>

#include "kv_common.cuh"
#include "pdl.cuh"

namespace kq {
namespace {

constexpr int kThreads = 128;      // forwards
constexpr int kGradThreads = 256;
constexpr int kMaxDim = 256;
// Blocks of an SM backwards: three have 85 registers a thread, which fp32's four values to a lane do with (16384 tokens of 20 fp32
// rows of 128: 103 us, with two 108) and bf16's eight do not (40 bf16 rows: 105 us with two, 270 with three).
template <typename T>
__host__ __device__ constexpr int grad_blocks_of(int nv) {
    return nv > 1 ? 1 : sizeof(T) == 4 ? 3 : 2;
}
constexpr int kManyRows = 36;      // of a token, see launch_mode
constexpr int kMaxBlocks = 512;    // that a workspace has room for the sums of
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
    int32_t parts, part;   // of a warp's tokens' rows, each of `part` looks at them
    float scale, eps;
    float* sums;       // backward: [blocks][2][dim] of weight gradients, or nullptr
};

// FAST: every row can be moved 16 bytes at a time, and has whole vectors; n: how much of a vector there is.
template <typename T, bool FAST>
struct Lane {
    static constexpr int E = 16 / sizeof(T);
    static __device__ __forceinline__ uint4 load(const T* p, int n) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if constexpr (FAST) {
            if (n > 0) u = *reinterpret_cast<const uint4*>(p);
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i < n) {
                    if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[i]);
                    else w[i / 2] |= static_cast<uint32_t>(__bfloat16_as_ushort(p[i])) << (16 * (i & 1));
                }
            u = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return u;
    }
    static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[E]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < E; ++i)
            x[i] = __uint_as_float(sizeof(T) == 4 ? w[i % 4] : i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    }
    static __device__ __forceinline__ void store(T* p, int n, const float (&x)[E]) {
        if constexpr (FAST) {
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
            if (n > 0) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (i < n) p[i] = static_cast<T>(x[i]);
        }
    }
};

// Two products, or products and sums, in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%2, %3};\n\t"
        "mov.b64 y, {%4, %5};\n\t"
        "mul.rn.f32x2 x, x, y;\n\t"
        "mov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%2, %3};\n\t"
        "mov.b64 y, {%4, %5};\n\t"
        "mov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\t"
        "mov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

template <int G>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A lane's share of a row, NV vectors l, l + G, .., and what it makes of it: with x_p the partner of x_i,
//     forwards  x_i c_i + x_p s_i,  c and s of cos, sin and the weights of the two,
//     backwards g_i c_i + g_p s_i,  of cos and sin alone (the transposed rotation).
// Values past the rotated ones have no partner: it counts as 0 whatever it holds.
template <typename T, int G, int NV, int MODE>
struct Share {
    static constexpr int E = 16 / sizeof(T);
    float c[NV][E], s[NV][E];
    int n[NV], turned[NV];     // values of a vector, and how many of them are rotated
    int l, step;               // vectors between partners (halves)

    __device__ __forceinline__ Share(int l_, int dim, int half) : l(l_), step(half / E) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            n[k] = min(E, max(0, dim - (l + k * G) * E));
            turned[k] = min(E, max(0, 2 * half - (l + k * G) * E));
        }
    }
    __device__ __forceinline__ int dim_of(int k, int e) const { return (l + k * G) * E + e; }
    // Whole warps call it. xch: the row in shared memory (odd halves).
    __device__ __forceinline__ void partners(const float (&x)[NV][E], float (&y)[NV][E], int half, float* xch) const {
        if constexpr (MODE == kPairs) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) y[k][e] = x[k][e ^ 1];
        } else if constexpr (MODE == kHalves) {
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
    }
    // c and s from a token's table; w: the weights, 1 where there are none, for what goes forwards.
    template <bool BACK>
    __device__ __forceinline__ void take(const float2* table, int half, const float (&w)[NV][E], float* xch) {
        float wp[NV][E];
        if constexpr (!BACK) partners(w, wp, half, xch);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int i = dim_of(k, e);
                const bool in = e < turned[k], second = MODE == kPairs ? e & 1 : i >= half;
                const float2 t = in ? table[MODE == kPairs ? i / 2 : second ? i - half : i] : make_float2(1.0f, 0.0f);
                c[k][e] = BACK ? t.x : t.x * w[k][e];
                s[k][e] = second != BACK ? t.y : -t.y;
                if constexpr (!BACK) s[k][e] = in ? s[k][e] * wp[k][e] : 0.0f;
            }
    }
    // FULL: every value is rotated.
    template <bool FULL>
    __device__ __forceinline__ void turn(float (&x)[NV][E], int half, float* xch) const {
        float y[NV][E];
        partners(x, y, half, xch);
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 a = make_float2(x[k][e], x[k][e + 1]), cc = make_float2(c[k][e], c[k][e + 1]);
                const float2 b = make_float2(FULL || e < turned[k] ? y[k][e] : 0.0f, FULL || e + 1 < turned[k] ? y[k][e + 1] : 0.0f);
                const float2 d = fma2(make_float2(s[k][e], s[k][e + 1]), b, mul2(cc, a));
                x[k][e] = d.x, x[k][e + 1] = d.y;
            }
    }
};

// cos and sin of the pairs of A tokens from t0 on, by a warp; a bit for each of them that is there and has a position.
template <int A, typename T>
__device__ __forceinline__ uint32_t fill_tables(const Rotate<T>& p, int64_t t0, float2* table) {
    const int lane = threadIdx.x & 31;
    bool is = lane < A && t0 + lane < p.tokens;
    int64_t mine = t0 + lane;   // position of token lane
    if (p.pos) {
        if (is) mine = p.pos[mine];
    } else if (p.start) {
#pragma unroll
        for (int a = 0; a < A; ++a) {
            const int b = kv_sequence_of_warp(p.start, p.batch, t0 + a);
            if (lane == a && is) {
                is = b >= 0;
                if (is) mine = p.first[b] + (mine - p.start[b]);
            }
        }
    }
    const uint32_t known = __ballot_sync(0xffffffffu, is);
    __syncwarp();   // the tables have had their last use
#pragma unroll
    for (int a = 0; a < A; ++a) {
        const uint64_t pos = static_cast<uint64_t>(__shfl_sync(0xffffffffu, mine, a));
        for (int j = lane; j < p.half; j += 32) {
            const int32_t turn = static_cast<int32_t>((pos * p.freq[j]) >> 32);
            float s, c;
            sincospif(static_cast<float>(turn) * 0x1p-31f, &s, &c);
            table[a * p.half + j] = make_float2(c * p.scale, s * p.scale);
        }
    }
    __syncwarp();
    return known;
}
// The 32 / G groups of lanes of a warp are of A tokens, and of as many rows of each as that leaves (A = 1 or 32 / G). They go
// through the rows together, queries, then keys, two looks at a time: an even number of looks at each.
__host__ __device__ constexpr int looks_at(int heads, int rows) { return (heads + 2 * rows - 1) / (2 * rows) * 2; }
__host__ __device__ constexpr int warp_floats(int mode, int g, int half, int dim) {   // of shared memory
    return (32 / g * 2 * half + (mode == kHalvesOdd ? 32 / g * dim : 0) + 1) & ~1;
}
// sum of x y
template <int NV, int E>
__device__ __forceinline__ float product_sum(const float (&x)[NV][E], const float (&y)[NV][E]) {
    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < E; e += 2) sum = fma2(make_float2(x[k][e], x[k][e + 1]), make_float2(y[k][e], y[k][e + 1]), sum);
    return sum.x + sum.y;
}
// x *= y
template <int NV, int E>
__device__ __forceinline__ void scale_by(float (&x)[NV][E], const float (&y)[NV][E]) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 d = mul2(make_float2(x[k][e], x[k][e + 1]), make_float2(y[k][e], y[k][e + 1]));
            x[k][e] = d.x, x[k][e + 1] = d.y;
        }
}
template <int NV, int E>
__device__ __forceinline__ void scale_by(float (&x)[NV][E], float y) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 d = mul2(make_float2(x[k][e], x[k][e + 1]), make_float2(y, y));
            x[k][e] = d.x, x[k][e + 1] = d.y;
        }
}
// x = y a + x
template <int NV, int E>
__device__ __forceinline__ void add_scaled(float (&x)[NV][E], const float (&y)[NV][E], float a) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 d = fma2(make_float2(y[k][e], y[k][e + 1]), make_float2(a, a), make_float2(x[k][e], x[k][e + 1]));
            x[k][e] = d.x, x[k][e + 1] = d.y;
        }
}
template <typename T, int NV, bool FAST, typename S>
__device__ __forceinline__ void unpack_weights(const T* w, const S& sh, float (&x)[NV][16 / sizeof(T)]) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (w) {
            Lane<T, FAST>::unpack(Lane<T, FAST>::load(w + sh.dim_of(k, 0), sh.n[k]), x[k]);
        } else {
#pragma unroll
            for (int e = 0; e < 16 / static_cast<int>(sizeof(T)); ++e) x[k][e] = 1.0f;
        }
    }
}

// A warp to a part of a token's rows. 28 warps on an SM: 24 or 20 leave too few loads in flight (32768 tokens of 40 bf16 rows of
// 128: 113, 118 and 118 us), 32 take too many registers (143).
template <typename T, int G, int NV, int MODE, bool FAST, int A>
__global__ void __launch_bounds__(kThreads, NV == 1 ? 7 : 4) qk_rotate_kernel(const Rotate<T> p) {
    using L = Lane<T, FAST>;
    constexpr int E = L::E, R = 32 / G;
    extern __shared__ __align__(16) float smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / G;
    const int64_t unit = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + warp, group = p.parts == 1 ? unit : unit / p.parts;
    constexpr int H = R / A;   // rows of a token in a look
    const int hsub = sub % H;
    const int64_t t0 = group * A, t = t0 + sub / H;
    if (t0 >= p.tokens) return;
    const bool mine = t < p.tokens;
    float* mem = smem + warp * warp_floats(MODE, G, p.half, p.dim);
    float2* table = reinterpret_cast<float2*>(mem);
    float* xch = mem + R * 2 * p.half + sub * p.dim;
    Share<T, G, NV, MODE> sh(lane % G, p.dim, p.half);
    const int queries = looks_at(p.s[0].heads, H), all = queries + looks_at(p.s[1].heads, H);
    const int first = static_cast<int>(unit - group * p.parts) * p.part, last = min(first + p.part, all);
    pdl_wait();
    pdl_launch_dependents();
    // the two looks that are fetched next, before the ones that are worked on
    int next = first;
    const T* src[2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int h = (side ? max(first - queries, 0) : first) * H + hsub;
        src[side] = p.s[side].x + t * p.s[side].x_token + h * p.s[side].x_head + sh.dim_of(0, 0);
    }
    uint4 raw[2][NV];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int k = 0; k < NV; ++k) raw[u][k] = make_uint4(0, 0, 0, 0);
    auto fetch = [&] {
        if (next >= last) return;
        const bool key = next >= queries;
        const int h = (key ? next - queries : next) * H + hsub, heads = key ? p.s[1].heads : p.s[0].heads;
        const int64_t head = H * (key ? p.s[1].x_head : p.s[0].x_head);
        const T* at = key ? src[1] : src[0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (mine && h + u * H < heads) {
#pragma unroll
                for (int k = 0; k < NV; ++k) raw[u][k] = L::load(at + u * head + k * G * E, sh.n[k]);
            }
        next += 2;
        if (key) src[1] = at + 2 * head;
        else src[0] = at + 2 * head;
    };
    fetch();
    const uint32_t known = fill_tables<A>(p, t0, table);
    if (known == 0) return;
    const bool is = known >> (sub / H) & 1;
    const float over = 1.0f / static_cast<float>(p.dim);
    const bool full = 2 * p.half == p.dim;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const Rows<T>& s = p.s[side];
        const int from = side ? max(first, queries) : first, to = side ? last : min(last, queries);
        if (from >= to) continue;
        const bool norm = s.w != nullptr;
        {
            float w[NV][E];
            unpack_weights<T, NV, FAST>(s.w, sh, w);
            sh.template take<false>(table + sub / H * p.half, p.half, w, xch);
        }
        int h = (side ? from - queries : from) * H;
        const int64_t head = H * s.o_head;
        T* dst = s.out + t * s.o_token + (h + hsub) * s.o_head + sh.dim_of(0, 0);
        for (int i = from; i < to; i += 2, h += 2 * H, dst += 2 * head) {
            float x[2][NV][E];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < NV; ++k) L::unpack(raw[u][k], x[u][k]);
            fetch();
            float r[2] = {1.0f, 1.0f};
            if (norm) {
#pragma unroll
                for (int u = 0; u < 2; ++u) r[u] = product_sum(x[u], x[u]);
#pragma unroll
                for (int u = 0; u < 2; ++u) r[u] = rsqrtf(fmaf(row_sum<G>(r[u]), over, p.eps));
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (h + u * H >= s.heads) break;
                if (full) sh.template turn<true>(x[u], p.half, xch);
                else sh.template turn<false>(x[u], p.half, xch);
                if (norm) scale_by(x[u], r[u]);
                if (is && h + u * H + hsub < s.heads) {
#pragma unroll
                    for (int k = 0; k < NV; ++k) L::store(dst + u * head + k * G * E, sh.n[k], x[u][k]);
                }
            }
        }
    }
}

// The same backwards. The warps go through units of a token's part in turn; the weights' gradients are summed in registers, then
// over the block's slots in order, then (rotate_sums_kernel) over the blocks in order.
template <typename T, int G, int NV, int MODE, bool FAST, int A>
__global__ void __launch_bounds__(kGradThreads, grad_blocks_of<T>(NV)) qk_rotate_grad_kernel(const Rotate<T> p) {
    using L = Lane<T, FAST>;
    constexpr int E = L::E, R = 32 / G, kWarps = kGradThreads / 32, kSlots = kWarps * R;
    extern __shared__ __align__(16) float smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / G;
    float* mem = smem + warp * warp_floats(MODE, G, p.half, p.dim);
    float2* table = reinterpret_cast<float2*>(mem);
    float* xch = mem + R * 2 * p.half + sub * p.dim;
    Share<T, G, NV, MODE> sh(lane % G, p.dim, p.half);
    constexpr int H = R / A;   // rows of a token in a look
    const int hsub = sub % H, tsub = sub / H;
    const int queries = looks_at(p.s[0].heads, H), looks = queries + looks_at(p.s[1].heads, H);
    const int64_t units = (p.tokens + A - 1) / A * p.parts, step = static_cast<int64_t>(gridDim.x) * kWarps;
    const bool full = 2 * p.half == p.dim;
    pdl_wait();
    pdl_launch_dependents();
    float w[NV][E], gw[2][NV][E];
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) gw[side][k][e] = w[k][e] = 0.0f;
    int weights_of = -1;
    const float over = 1.0f / static_cast<float>(p.dim);
    // the two looks that are fetched next, before the ones that are worked on, across units
    int64_t next_unit = static_cast<int64_t>(blockIdx.x) * kWarps + warp, next_t = 0;
    int next = 0, next_last = 0;
    auto enter = [&] {
        if (next_unit >= units) return;
        const int64_t group = p.parts == 1 ? next_unit : next_unit / p.parts;
        next_t = group * A + tsub;
        next = static_cast<int>(next_unit - group * p.parts) * p.part;
        next_last = min(next + p.part, looks);
    };
    uint4 rx[2][NV], rg[2][NV];
    auto fetch = [&] {
        if (next_unit >= units) return;
        const int side = next >= queries, h0 = (side ? next - queries : next) * H + hsub;
        const Rows<T>& s = p.s[side];
        const T* gy = s.gy + next_t * s.g_token + h0 * s.g_head + sh.dim_of(0, 0);
        const T* x = s.x + next_t * s.x_token + h0 * s.x_head + sh.dim_of(0, 0);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool here = next_t < p.tokens && h0 + u * H < s.heads;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                // a row that is not there: a gradient of 0, of a row of ones, whose r is finite
                constexpr uint32_t kOne = sizeof(T) == 4 ? 0x3F800000u : 0x3F803F80u;
                rx[u][k] = make_uint4(kOne, kOne, kOne, kOne);
                rg[u][k] = make_uint4(0, 0, 0, 0);
                if (here) rg[u][k] = L::load(gy + u * H * s.g_head + k * G * E, sh.n[k]);
                if (here && s.w) rx[u][k] = L::load(x + u * H * s.x_head + k * G * E, sh.n[k]);
            }
        }
        next += 2;
        if (next >= next_last) {
            next_unit += step;
            enter();
        }
    };
    int64_t unit = next_unit;
    enter();
    fetch();
    for (; unit < units; unit += step) {
        const int64_t group = p.parts == 1 ? unit : unit / p.parts, t = group * A + tsub;
        const int first = static_cast<int>(unit - group * p.parts) * p.part, last = min(first + p.part, looks);
        const bool is = fill_tables<A>(p, group * A, table) >> tsub & 1;
        sh.template take<true>(table + tsub * p.half, p.half, w, xch);
        for (int i = first; i < last; i += 2) {
            float g[2][NV][E], x[2][NV][E];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    L::unpack(rg[u][k], g[u][k]);
                    L::unpack(rx[u][k], x[u][k]);
                }
            fetch();
            const int side = i >= queries, h0 = (side ? i - queries : i) * H + hsub;
            const Rows<T>& s = p.s[side];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (full) sh.template turn<true>(g[u], p.half, xch);
                else sh.template turn<false>(g[u], p.half, xch);
            }
            if (s.w) {
                if (side != weights_of) {
                    unpack_weights<T, NV, FAST>(s.w, sh, w);
                    weights_of = side;
                }
                float sum[2], dot[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    // x g first, for the weights; its sum with w is the mean's
                    sum[u] = product_sum(x[u], x[u]);
                    float xg[NV][E];
#pragma unroll
                    for (int k = 0; k < NV; ++k)
#pragma unroll
                        for (int e = 0; e < E; ++e) xg[k][e] = x[u][k][e];
                    scale_by(xg, g[u]);
                    dot[u] = product_sum(xg, w);
                    sum[u] = row_sum<G>(sum[u]);
                    dot[u] = row_sum<G>(dot[u]);
                    const float r = rsqrtf(fmaf(sum[u], over, p.eps)), f = dot[u] * over * r * r;
                    if (is) {   // rows that are not there count as 0
                        if (side) add_scaled(gw[1], xg, r);
                        else add_scaled(gw[0], xg, r);
                    }
                    scale_by(g[u], w);
                    add_scaled(g[u], x[u], -f);
                    scale_by(g[u], r);
                }
            }
            T* dst = s.out + t * s.o_token + h0 * s.o_head + sh.dim_of(0, 0);
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (is && h0 + u * H < s.heads) {
#pragma unroll
                    for (int k = 0; k < NV; ++k) L::store(dst + u * H * s.o_head + k * G * E, sh.n[k], g[u][k]);
                }
        }
    }
    if (!p.sums) return;
    float* all = smem;   // [kSlots][dim]
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < sh.n[k]) all[(warp * R + sub) * p.dim + sh.dim_of(k, e)] = gw[side][k][e];
        __syncthreads();
        for (int d = threadIdx.x; d < p.dim; d += kGradThreads) {
            float sum = 0.0f;
            for (int q = 0; q < kSlots; ++q) sum += all[q * p.dim + d];
            if (KQ_IN_RANGE(blockIdx.x, kMaxBlocks)) p.sums[(static_cast<int64_t>(blockIdx.x) * 2 + side) * p.dim + d] = sum;
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

int64_t grad_blocks(int64_t tokens) { return std::min<int64_t>(tokens, kMaxBlocks); }

template <typename T, int G, int NV, int MODE, bool FAST, int A>
kq_status launch(Rotate<T>& p, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    constexpr int R = 32 / G;
    const int64_t looks = looks_at(p.s[0].heads, R / A) + looks_at(p.s[1].heads, R / A), groups = cdiv(p.tokens, A);
    const int64_t warps = static_cast<int64_t>(num_sms()) * 16;
    // a token's rows go to several warps where tokens are few
    const int64_t parts = std::max<int64_t>(1, std::min(looks / 2, warps / groups));
    p.part = static_cast<int32_t>(cdiv(looks / 2, parts) * 2);
    p.parts = static_cast<int32_t>(cdiv(looks, p.part));
    const size_t floats = warp_floats(MODE, G, p.half, p.dim);
    const int64_t units = groups * p.parts;
    if (!back) {
        KQ_CUDA(launch_after(qk_rotate_kernel<T, G, NV, MODE, FAST, A>, dim3(static_cast<unsigned>(cdiv(units, kThreads / 32))),
                             dim3(kThreads), kThreads / 32 * floats * sizeof(float), stream, p));
        count_launch();
        return KQ_OK;
    }
    constexpr int kWarps = kGradThreads / 32;
    const int64_t fit = static_cast<int64_t>(num_sms()) * grad_blocks_of<T>(NV);
    const int blocks = static_cast<int>(std::min({grad_blocks(p.tokens), cdiv(units, kWarps), fit}));
    size_t smem = kWarps * floats * sizeof(float);
    if (p.sums) smem = std::max(smem, kWarps * R * p.dim * sizeof(float));
    KQ_CUDA(launch_after(qk_rotate_grad_kernel<T, G, NV, MODE, FAST, A>, dim3(blocks), dim3(kGradThreads), smem, stream, p));
    count_launch();
    if (p.sums) {
        KQ_CUDA(launch_after(rotate_sums_kernel, dim3(static_cast<unsigned>(cdiv(p.dim, 32)), 2), dim3(1024), 0, stream,
                             static_cast<const float*>(p.sums), blocks, static_cast<int>(p.dim), gqw, gkw));
        count_launch();
    }
    return KQ_OK;
}

template <typename T, int G, int NV>
kq_status launch_mode(Rotate<T>& p, bool fast, bool pairs, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    constexpr int R = 32 / G;
    // A token to a warp where it has many rows (32768 tokens of 40 bf16 rows of 128: 119 us, two tokens abreast 123; 16384
    // backwards 105 and 107), else a token to each group of lanes, which are all at work whatever the rows (30000 tokens of 16 rows: 48
    // and 46 us, backwards 80 and 78; 52708 of 4 + 2 rows of 64: 45 and 19, 75 and 38; of 1 + 1 of 128: 47 and 26, 78 and 43).
    const bool one = p.s[0].heads + p.s[1].heads >= kManyRows;
    if (!fast) {   // rows of any alignment: one value at a time, partners through shared memory where they are not neighbours
        return pairs ? launch<T, G, NV, kPairs, false, R>(p, back, gqw, gkw, stream)
                     : launch<T, G, NV, kHalvesOdd, false, R>(p, back, gqw, gkw, stream);
    }
    if (pairs)
        return one ? launch<T, G, NV, kPairs, true, 1>(p, back, gqw, gkw, stream) : launch<T, G, NV, kPairs, true, R>(p, back, gqw, gkw, stream);
    if (p.half % (16 / sizeof(T)) == 0)
        return one ? launch<T, G, NV, kHalves, true, 1>(p, back, gqw, gkw, stream) : launch<T, G, NV, kHalves, true, R>(p, back, gqw, gkw, stream);
    return launch<T, G, NV, kHalvesOdd, true, R>(p, back, gqw, gkw, stream);
}
kq_status launch_dim(Rotate<__nv_bfloat16>& p, bool fast, bool pairs, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    if (p.dim <= 64) return launch_mode<__nv_bfloat16, 8, 1>(p, fast, pairs, back, gqw, gkw, stream);
    if (p.dim <= 128) return launch_mode<__nv_bfloat16, 16, 1>(p, fast, pairs, back, gqw, gkw, stream);
    return launch_mode<__nv_bfloat16, 32, 1>(p, fast, pairs, back, gqw, gkw, stream);
}
kq_status launch_dim(Rotate<float>& p, bool fast, bool pairs, bool back, float* gqw, float* gkw, cudaStream_t stream) {
    if (p.dim <= 64) return launch_mode<float, 16, 1>(p, fast, pairs, back, gqw, gkw, stream);
    if (p.dim <= 128) return launch_mode<float, 32, 1>(p, fast, pairs, back, gqw, gkw, stream);
    return launch_mode<float, 32, 2>(p, fast, pairs, back, gqw, gkw, stream);
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
    p.sums = sums;
    return launch_dim(p, !((bits | dim * sizeof(T)) & 15u), r->interleaved != 0, gq != nullptr, gqw, gkw, stream);
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
        if ((out[i]->token_stride == 0 && T > 1) || (out[i]->head_stride == 0 && out[i]->heads > 1)) {
            set_error("%s: rows of an output must not share their place", who);
            return KQ_ERR_INVALID_ARG;
        }
        if (w[i] && (!(eps >= 0.0f) || !(eps - eps == 0.0f) || (reinterpret_cast<uintptr_t>(w[i]) & (es - 1)))) {
            set_error("%s: norms need eps >= 0 and weights aligned to their type", who);
            return KQ_ERR_INVALID_ARG;
        }
    }
    return KQ_OK;
}

// A side's warps do not wait for the other's: neither output may be the other one, nor what the other side reads (x, and backwards g).
kq_status check_places(const char* who, const kq_heads* const (&out)[2], const kq_heads* const (&x)[2], const kq_heads* const (&g)[2]) {
    if (!out[1]) return KQ_OK;
    bool same = out[0]->data == out[1]->data;
    for (int i = 0; i < 2; ++i) same = same || (x[1 - i] && out[i]->data == x[1 - i]->data) || (g[1 - i] && out[i]->data == g[1 - i]->data);
    if (!same) return KQ_OK;
    set_error("%s: the outputs must not be each other or an input of each other's", who);
    return KQ_ERR_INVALID_ARG;
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
    KQ_TRY(check_places("kq_qk_rotate", {q_out, k_out}, {q, k}, {nullptr, nullptr}));
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
    KQ_TRY(check_places(who, {q_out, k_out}, {q_weight ? q : nullptr, k_weight ? k : nullptr}, {gq, gk}));
    if (gq_weight && gq_weight == gk_weight) {
        set_error("%s: the weights' gradients must not be each other", who);
        return KQ_ERR_INVALID_ARG;
    }
    float* s = sums ? static_cast<float*>(ws) : nullptr;
    if (dtype == KQ_BF16)
        return run<__nv_bfloat16>(r, T, dim, q, k, gq, gk, q_out, k_out, q_weight, k_weight, eps, gq_weight, gk_weight, s,
                                  stream);
    return run<float>(r, T, dim, q, k, gq, gk, q_out, k_out, q_weight, k_weight, eps, gq_weight, gk_weight, s, stream);
}
