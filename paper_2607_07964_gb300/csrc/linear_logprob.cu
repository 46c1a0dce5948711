// kq_linear_logprobs and kq_linear_logprobs_grad: log probabilities straight from hidden states, no logits kept.
//
// Mathematics. z = x W^T for T rows of hidden states x [T][d] and a head W [V][d]. For each row
//     lse = ln sum_v e^(z_v),  logp = z_y - lse,  entropy = -sum_v p_v ln p_v,  p_v = e^(z_v - lse).
// A tile of logits leaves, for each row and 64 columns, the maximum m, Z = sum 2^t and S = sum 2^t t with
// t = log2(e) (z - m), and the target's logit where it has it. (The difference first: it is exact near the maximum, whatever
// its size.) Joined: M = max m, lse = M + ln Z, entropy = (log2 Z - S / Z) ln 2.
// Gradient of sum_t (g logp + h entropy): the logits' is
//     D_v = g (delta(v, y) - p_v) - h p_v (ln p_v + entropy),   gx = D W,  gW = D^T x.
// The vocabulary goes in pieces: D of a piece (logits computed again, from the log-sums) is held in bf16, read for
// both products, and overwritten. bf16 has D's range and moves a sum of its terms by 2^-9 of the terms' size at
// most, the size of the outputs' own rounding.
//
// What bounds it: the tensor cores where there are many rows (2 T V d operations a product), the bytes of W where there
// are few. Layout: a cluster of two CTAs on two SMs holds a 256 x 256 tile (tcgen05 cta_group::2, each SM the
// accumulator of 128 rows in tensor memory and half of each operand in shared memory); one warp issues the TMA
// loads of 64-wide boxes into a ring, one the products, 16 read accumulators and work on them while the
// next chunk's products run into the other accumulator. Both operand layouts come from the same boxes: 64 of the
// contiguous dimension by 64 rows, 128-byte swizzle, is 64 rows of 64 k for a K-major operand and 64 k of 64 rows for
// an MN-major one. A launch carries the tiles of gx and gW of one piece and those of D of the next, so that the
// clusters stay busy while the counts of each do not divide by the clusters.
//   An accumulator is added to an fp32 sum in registers every kDrain slabs of 64: the tensor cores truncate their
// sums, 2^-24.5 of them for each 16 products. (4096 x 64000 x 4096 logits: 1270, 1220, 1160 to 1210 us with 8, 16, 32 slabs; the
// log-sums are 2e-7 and 4e-7 off with 8 and 16.)
//
// Measured: logits of 4096 x 128000 x 4096 2440 us, 1.76 PFLOP/s under the power cap (one launch of 4096 x 32000 x 4096 by itself
// 543 us, 1.98); both gradients of 4096 x 128000 x 2048 4.11 ms, 1.57 PFLOP/s.
#include <algorithm>
#include <atomic>
#include <cstring>

#include <cuda_bf16.h>

#include "kq_common.cuh"
#include "pdl.cuh"
#include "trail_tc.cuh"

namespace kq {
namespace {

constexpr int BM = 256, BN = 256;                // tile of a pair
constexpr int BK = 64;                           // of a slab
constexpr int kBox = 64 * 64 * 2;                // bytes
constexpr int kStage = 4 * kBox;                 // a CTA's 128 rows of A and 128 of B
constexpr int kStages = 5;
constexpr int kOutBox = 32 * 64 * 2;             // bytes of a warp's 32 rows by 64 columns of results
constexpr int kThreads = 640;                    // a warpgroup for loads and products, 16 warps for results
// Registers of a thread: the launch gives all 96 (what 65536 leave 640 threads); results need a row's 64 sums and more.
constexpr int kIssueRegs = 64, kResultRegs = 104;
static_assert(128 * kIssueRegs + 512 * kResultRegs <= kThreads * 96, "more registers than the block was launched with");
constexpr int kSmem = kStages * kStage + 16 * kOutBox + 1024 + 256;
constexpr int kDrainLogits = 16, kDrainGrads = 32, kDrainThin = 8;   // slabs
constexpr int kTileCost = 1;                     // what beginning and ending a tile costs, in slabs
constexpr int kBand = 16;                        // row tiles that go through the vocabulary together
constexpr int64_t kPiece = 1 << 26;              // elements of D that a piece holds, about
constexpr int64_t kLeastPiece = 1024;            // columns
constexpr int64_t kMostParts = 1 << 24;          // sums of 64 logits that scoring holds at once, of 4096 rows at least
constexpr int kMostPairs = 96;                   // clusters that a launch with tiles of several sizes has
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kNone = -1.0e30f;                // t of a logit that cannot occur: 2^t = 0 and 0 t a number

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Whether p holds in all 256 threads of the eight result warps; a barrier for them.
__device__ __forceinline__ bool named_all(bool p) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred a, b;\n\t"
        "setp.ne.u32 a, %1, 0;\n\t"
        "barrier.red.and.pred b, 1, 256, a;\n\t"
        "selp.u32 %0, 1, 0, b;\n\t}"
        : "=r"(r)
        : "r"(static_cast<uint32_t>(p))
        : "memory");
    return r != 0;
}
// The bounded waits of kq_common.cuh in which the hardware holds the thread back for up to kHold at a time, not for its
// own short while: the result warps wait for most of a tile, and polling takes issue slots and power from the products.
constexpr uint32_t kHold = 20000;   // ns
template <bool CLUSTER>
__device__ __forceinline__ bool held_try(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    if constexpr (CLUSTER)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity), "r"(kHold)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity), "r"(kHold)
            : "memory");
    return ok != 0;
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool held_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
    if (held_try<CLUSTER>(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (uint32_t it = 0; it < kWaitLimitIters; ++it) {
        if (held_try<CLUSTER>(bar, parity)) return true;
        if (*abort) return false;
        if (global_timer_ns() - t0 > kWaitLimitNs) break;
    }
    *abort = 1;
    return false;
}
// 16 consecutive fp32 columns of the calling warp's 32 lanes of tensor memory.
__device__ __forceinline__ void tmem_ld16(uint32_t at, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
// 32 bytes, on a 32-byte boundary.
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}

// Two sums, products, or products and sums, in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\t"
        "mov.b64 x, {%2, %3};\n\t"
        "mov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 x, x, y;\n\t"
        "mov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
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

// The sums over one set of logits, against their maximum, joined with those over another: against the larger maximum.
struct Sums {
    float m, z, s;
    __device__ __forceinline__ void join(float m2, float z2, float s2) {
        const float top = max_nan(m, m2);
        if (top == -INFINITY) return;
        const float a = (m - top) * kLog2e, b = (m2 - top) * kLog2e, fa = ex2(a), fb = ex2(b);
        // 2^b (s + b z); one against -infinity has none
        s = (fa > 0.0f || a != a ? fa * fmaf(a, z, s) : 0.0f) + (fb > 0.0f || b != b ? fb * fmaf(b, z2, s2) : 0.0f);
        z = fa * z + fb * z2;
        m = top;
    }
};

enum Kind { kScore, kDelta, kGx, kGw };

struct Job {
    int64_t T, V, d;
    const int64_t* target;
    // score
    float4* part;              // [T][parts]: m, Z, S of 64 columns
    float* zt;                 // [T] the target's logit
    int32_t parts;
    // gradient
    const float *lse, *entropy, *g_logp, *g_entropy;
    __nv_bfloat16* delta;      // of the piece that this launch makes, [T][ld_delta]
    int64_t ld_delta;
    int64_t v_main, v_prod;    // the first column of the piece whose logits, whose products are computed
    int64_t w_main, w_prod;    // and its width
    float* sum;                // [splits][T][d]: gx so far
    bool first, last;          // no gx so far; this launch finishes it
    bool turned;               // D is by columns: a row of tokens for each row of W
    bool gw;                   // few rows: gW is asked for
    int32_t splits, split_slabs;
    int32_t m_main, n_main, m_prod, n_d;   // tiles of the rows, of the columns, of the rows again, of d
    int32_t d_slabs, row_slabs, prod_slabs;   // slabs of d, of the rows, of the piece whose products are computed
    int32_t t_gx, t_gw, tiles;             // tiles of each, in this order, and in all
    int32_t first_main[kMostPairs + 1];    // with products: a pair's logits' tiles are from its entry to the next's
    int* info;
};

struct Tile {
    int kind;
    int m0, n0;      // of the tile, in its operands
    int ka, kb;      // where K begins in A, in B
    int slabs, split;
};
__device__ __forceinline__ Tile tile_at(const Job& j, int t, int main_kind) {
    Tile a;
    a.split = 0;
    if (t < j.t_gx) {
        const int each = j.m_prod * j.n_d;
        a.kind = kGx;
        a.split = t / each;
        t -= a.split * each;
        const int m = t / j.n_d;
        a.m0 = m * BM;
        a.n0 = (t - m * j.n_d) * BN;
        a.ka = a.split * j.split_slabs * BK;
        a.kb = static_cast<int>(j.v_prod) + a.ka;
        a.slabs = min(j.split_slabs, j.prod_slabs - a.split * j.split_slabs);
        return a;
    }
    t -= j.t_gx;
    if (t < j.t_gw) {
        a.kind = kGw;
        const int m = t / j.n_d;
        a.m0 = m * BM;
        a.n0 = (t - m * j.n_d) * BN;
        a.ka = a.kb = 0;
        a.slabs = j.row_slabs;
        return a;
    }
    t -= j.t_gw;
    // bands of row tiles, each through all columns, rows first
    a.kind = main_kind;
    const int band = t / (kBand * j.n_main), rows = min(kBand, j.m_main - band * kBand);
    t -= band * kBand * j.n_main;
    const int n = t / rows;
    a.m0 = (band * kBand + t - n * rows) * BM;
    a.n0 = n * BN;
    a.ka = a.kb = 0;
    a.slabs = j.d_slabs;
    return a;
}

// Waits for a phase that the CTA's own earlier work ends, whatever has been given up.
__device__ __forceinline__ void wait_quiet(uint64_t* bar, uint32_t parity) {
    int none = 0;
    held_wait(bar, parity, &none);
}
__host__ __device__ __forceinline__ int round_tile(int rd, int pair, int pairs) {
    return rd * pairs + ((rd & 1) ? pairs - 1 - pair : pair);
}
// A pair's tiles: of the products every pairs-th, back and forth; then of the logits a run that evens the pairs' work out. Where
// there are no products every pairs-th of the logits, so that the pairs share rows of W.
struct Walk {
    int pair, pairs, dealt, run, count;
    __device__ __forceinline__ Walk(const Job& j, int pair_, int pairs_) : pair(pair_), pairs(pairs_) {
        const int deal = j.t_gx + j.t_gw ? j.t_gx + j.t_gw : j.tiles, whole = deal / pairs;
        dealt = whole + (round_tile(whole, pair, pairs) < deal ? 1 : 0);
        run = deal + (deal < j.tiles ? j.first_main[pair] : 0);
        count = dealt + (deal < j.tiles ? j.first_main[pair + 1] - j.first_main[pair] : 0);
    }
    __device__ __forceinline__ int at(int n) const { return n < dealt ? round_tile(n, pair, pairs) : run + n - dealt; }
};

// m, Z and S of 64 logits of a row, and the target's logit.
__device__ __forceinline__ Sums score_row(const Job& j, float (&x)[64], int64_t row, int64_t col) {
    Sums a = {-INFINITY, 0.0f, 0.0f};
    const int64_t left = j.V - col;
    if (row >= j.T || left <= 0) return a;
    if (left < 64) {
#pragma unroll
        for (int i = 0; i < 64; ++i)
            if (i >= left) x[i] = -INFINITY;
    }
    const int64_t y = j.target[row] - col;
    if (y >= 0 && y < min(left, static_cast<int64_t>(64))) {
        float z = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i)
            if (i == y) z = x[i];
        j.zt[row] = z;
    }
    a.m = x[0];
#pragma unroll
    for (int i = 1; i < 64; ++i) a.m = max_nan(a.m, x[i]);
    const float ref = a.m == -INFINITY ? 0.0f : a.m;
    float2 z[2] = {}, s[2] = {};
    const float2 less = make_float2(-ref, -ref), log2e = make_float2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < 64; i += 2) {
        float2 t = mul2(add2(make_float2(x[i], x[i + 1]), less), log2e);
        t.x = fmaxf(t.x, kNone), t.y = fmaxf(t.y, kNone);
        const float2 e = make_float2(ex2(t.x), ex2(t.y));
        z[i / 2 & 1] = add2(z[i / 2 & 1], e);
        s[i / 2 & 1] = fma2(e, t, s[i / 2 & 1]);
    }
    a.z = (z[0].x + z[0].y) + (z[1].x + z[1].y);
    a.s = (s[0].x + s[0].y) + (s[1].x + s[1].y);
    return a;
}

// What a logit z contributes to D but for the target's own share: -p (g + ge (ln p + h)).
__device__ __forceinline__ float delta_of(float z, float lse, float g, float ge, float h) {
    const float lp = z - lse, p = ex2(lp * kLog2e);
    return p > 0.0f ? -p * fmaf(ge, lp + h, g) : p == p ? 0.0f : p;
}

// 64 columns of a warp's 32 rows to a bf16 matrix by way of shared memory: a box of 128-byte lines, swizzled, a line to a lane.
// put_part: columns 8 FROM .. 8 TO, value(i) is this lane's column i. What lies outside the matrix (rows x cols) is left out.
__device__ __forceinline__ void put_begin() {
    if ((threadIdx.x & 31) == 0) bulk_wait_read0();   // the last results have left the box
    __syncwarp();
}
template <int FROM, int TO, typename F>
__device__ __forceinline__ void put_part(uint8_t* box, F value) {
    const int lane = threadIdx.x & 31;
    uint4* line = reinterpret_cast<uint4*>(box + lane * 128);
#pragma unroll
    for (int c = FROM; c < TO; ++c) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = pack_bf16(value(8 * c + 2 * k), value(8 * c + 2 * k + 1));
        line[c ^ (lane & 7)] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ void put_end(uint8_t* box, const CUtensorMap* map, int64_t row0, int64_t rows, int64_t col0, int64_t cols) {
    fence_proxy_async();
    __syncwarp();
    if ((threadIdx.x & 31) == 0 && row0 < rows && col0 < cols) {
        tma_store_2d(map, box, static_cast<int>(col0), static_cast<int>(row0));
        bulk_commit();
    }
}
template <typename F>
__device__ __forceinline__ void put_rows(uint8_t* box, const CUtensorMap* map, int64_t row0, int64_t rows, int64_t col0, int64_t cols,
                                         F value) {
    if (row0 >= rows || col0 >= cols) return;   // the same for the warp
    put_begin();
    put_part<0, 8>(box, value);
    put_end(box, map, row0, rows, col0, cols);
}

// D of 64 logits of a row, zeros from the vocabulary's end on.
__device__ __forceinline__ void delta_rows(const Job& j, const float (&x)[64], uint8_t* box, const CUtensorMap* map, int64_t row0,
                                           int64_t col) {
    const int64_t row = row0 + (threadIdx.x & 31), left = j.V - j.v_main - col;
    const bool is = row < j.T;
    const int64_t y = is ? j.target[row] : -1;
    const float lse = is ? j.lse[row] : -INFINITY, g = y >= 0 && y < j.V ? j.g_logp[row] : 0.0f;
    const float ge = is && j.g_entropy ? j.g_entropy[row] : 0.0f, h = is && j.g_entropy ? j.entropy[row] : 0.0f;
    const bool none = lse == -INFINITY;
    const int64_t at = y - j.v_main - col;
    const int here = at >= 0 && at < 64 && y < j.V && !none ? static_cast<int>(at) : -1;
    const int end = none ? 0 : static_cast<int>(max(static_cast<int64_t>(0), min(left, static_cast<int64_t>(64))));
    put_rows(box, map, row0, j.T, col, j.ld_delta, [&](int i) {
        const float q = i < end ? delta_of(x[i], lse, g, ge, h) : 0.0f;
        return i == here ? q + g : q;
    });
}

// gx so far plus 64 values of a row.
__device__ __forceinline__ void add_gx(const Job& j, float (&x)[64], int split, uint8_t* box, const CUtensorMap* map, int64_t row0,
                                       int64_t col) {
    const int64_t row = row0 + (threadIdx.x & 31);
    const bool is = row < j.T && col < j.d;
    float* sum = j.sum + (static_cast<int64_t>(split) * j.T + row) * j.d + col;
    if (!j.first && is) {
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            if (col + 4 * c >= j.d) break;
            const float4 o = *reinterpret_cast<const float4*>(sum + 4 * c);
            x[4 * c] += o.x, x[4 * c + 1] += o.y, x[4 * c + 2] += o.z, x[4 * c + 3] += o.w;
        }
    }
    if (j.last) {
        put_rows(box, map, row0, j.T, col, j.d, [&](int i) { return x[i]; });
        return;
    }
    if (!is) return;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        if (col + 8 * c >= j.d) break;
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(x[8 * c + k]);
        store32(sum + 8 * c, w);
    }
}

// Clusters walk the tiles of a job. MAIN: kScore or kDelta; only kDelta's launches have gradient tiles.
template <int MAIN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_tile_kernel(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
                   const __grid_constant__ CUtensorMap md, const __grid_constant__ CUtensorMap out_d,
                   const __grid_constant__ CUtensorMap out_x, const __grid_constant__ CUtensorMap out_w, const __grid_constant__ Job j) {
    const uint32_t rank = cluster_ctarank();
    const Walk walk(j, static_cast<int>(blockIdx.x >> 1), static_cast<int>(gridDim.x >> 1));
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* boxes = smem + kStages * kStage;   // of the result warps
    uint64_t* full = reinterpret_cast<uint64_t*>(boxes + 16 * kOutBox);
    uint64_t* empty = full + kStages;
    uint64_t* tfull = empty + kStages;
    uint64_t* tempty = tfull + 2;
    uint64_t* mma_done = tempty + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tfull[b], 1);
            mbar_init(&tempty[b], 32);   // 16 result warps in each CTA
        }
        mbar_init(mma_done, 1);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, 2 * BN);
        tmem_relinquish_pair();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&mx);
        tma_prefetch_desc(&mw);
        if (MAIN == kDelta) tma_prefetch_desc(&md);
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();   // both CTAs' barriers are there before one is signalled from the other
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();   // nothing before this reads or writes global memory
    pdl_launch_dependents();
    const uint32_t full0 = mapa_shared(smem_u32(full), 0), tempty0 = mapa_shared(smem_u32(tempty), 0);   // CTA 0's

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
        // ---- loads, each CTA its own half
        if (warp == 0 && lane == 0) {
            int k = 0;
            bool ok = true;
            for (int i = 0; i < walk.count && ok; ++i) {
                const Tile a = tile_at(j, walk.at(i), MAIN);
                const bool a_mn = a.kind == (j.turned ? kGx : kGw), b_mn = a.kind == kGx || a.kind == kGw;
                const CUtensorMap* ma = a.kind == kGx || a.kind == kGw ? &md : &mx;
                const CUtensorMap* mb = a.kind == kGw ? &mx : &mw;
                const int m = a.m0 + 128 * static_cast<int>(rank);
                const int n = a.n0 + 128 * static_cast<int>(rank) + (a.kind == MAIN ? static_cast<int>(j.v_main) : 0);
                for (int s = 0; s < a.slabs; ++s, ++k) {
                    const int st = k % kStages;
                    if (!held_wait(&empty[st], (static_cast<uint32_t>(k / kStages) & 1u) ^ 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_arrive_expect_tx(&full[st], 2 * kStage);
                    uint8_t* base = smem + st * kStage;
                    const uint32_t bar = full0 + static_cast<uint32_t>(st * 8);
                    const int ka = a.ka + s * BK, kb = a.kb + s * BK;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        tma_load_2d_pair(base + i * kBox, ma, bar, a_mn ? m + 64 * i : ka, a_mn ? ka : m + 64 * i);
                        tma_load_2d_pair(base + (2 + i) * kBox, mb, bar, b_mn ? n + 64 * i : kb, b_mn ? kb : n + 64 * i);
                    }
                }
            }
            // the last slabs have been used by the products, so they have landed
            for (int i = (k > kStages ? k - kStages : 0); i < k; ++i)
                wait_quiet(&empty[i % kStages], static_cast<uint32_t>(i / kStages) & 1u);
        }
        // ---- products, CTA 0 for both
        if (warp == 1 && lane == 0) {
            if (rank == 0) {
                int k = 0, cc = 0;
                bool ok = true;
                for (int i = 0; i < walk.count && ok; ++i) {
                    const Tile a = tile_at(j, walk.at(i), MAIN);
                    const bool a_mn = a.kind == (j.turned ? kGx : kGw), b_mn = a.kind == kGx || a.kind == kGw;
                    const uint32_t idesc = (idesc_bf16_mn_major(BM, BN) & ~(3u << 15)) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
                    // to the next 16 of K: 32 bytes along swizzled rows, or 16 rows of 128 bytes
                    const uint32_t a_step = a_mn ? 2048 : 32, b_step = b_mn ? 2048 : 32;
                    const int drain = a.kind == MAIN ? kDrainLogits : kDrainGrads;
                    for (int s0 = 0; s0 < a.slabs && ok; s0 += drain, ++cc) {
                        const int buf = cc & 1;
                        if (!held_wait<true>(&tempty[buf], ((static_cast<uint32_t>(cc) >> 1) & 1u) ^ 1u, abort_flag)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        const uint32_t dt = tmem + static_cast<uint32_t>(buf * BN);
                        const int s1 = min(a.slabs, s0 + drain);
                        for (int s = s0; s < s1; ++s, ++k) {
                            const int st = k % kStages;
                            if (!held_wait(&full[st], static_cast<uint32_t>(k / kStages) & 1u, abort_flag)) {
                                ok = false;
                                break;
                            }
                            tc_fence_after();
                            const uint32_t sa = smem_u32(smem + st * kStage), sb = sa + 2 * kBox;
#pragma unroll
                            for (int q = 0; q < BK / 16; ++q)
                                mma_pair(dt, smem_desc_sw128(sa + q * a_step, kBox, 1024), smem_desc_sw128(sb + q * b_step, kBox, 1024),
                                         idesc, (s > s0 || q > 0) ? 1u : 0u);
                            tc_commit_pair(&empty[st]);
                        }
                        if (ok) tc_commit_pair(&tfull[buf]);
                    }
                }
                tc_commit_pair(mma_done);
            }
            wait_quiet(mma_done, 0);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kResultRegs));
        // ---- results: a thread has 64 columns of one of the CTA's 128 rows
        const int q = warp & 3, h = (warp - 4) >> 2;
        uint8_t* box = boxes + (warp - 4) * kOutBox;
        int cc = 0;
        bool ok = true;
        for (int i = 0; i < walk.count && ok; ++i) {
            const Tile a = tile_at(j, walk.at(i), MAIN);
            const int drain = a.kind == MAIN ? kDrainLogits : kDrainGrads;
            float x[64];
            for (int s0 = 0; s0 < a.slabs; s0 += drain, ++cc) {
                const int buf = cc & 1;
                ok = held_wait(&tfull[buf], (static_cast<uint32_t>(cc) >> 1) & 1u, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const uint32_t at = tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(buf * BN + h * 64);
                if (s0 == 0) {
#pragma unroll
                    for (int p = 0; p < 2; ++p) tmem_ld32(at + p * 32, reinterpret_cast<float(&)[32]>(x[p * 32]));
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        float v[16];
                        tmem_ld16(at + p * 16, v);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[p * 16 + i] += v[i];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(tempty0 + static_cast<uint32_t>(buf * 8));
            }
            if (!ok) break;
            const int64_t row0 = a.m0 + 128 * static_cast<int64_t>(rank) + q * 32, col = a.n0 + h * 64;
            if (MAIN == kScore) {
                const Sums sums = score_row(j, x, row0 + lane, col);
                if (row0 + lane < j.T && col < j.V && KQ_IN_RANGE(a.n0 / 64 + h, j.parts))
                    j.part[(row0 + lane) * j.parts + a.n0 / 64 + h] = make_float4(sums.m, sums.z, sums.s, 0.0f);
            } else if (a.kind == kDelta) {
                delta_rows(j, x, box, &out_d, row0, col);
            } else if (a.kind == kGx) {
                add_gx(j, x, a.split, box, &out_x, row0, col);
            } else {
                put_rows(box, &out_w, j.v_prod + row0, j.V, col, j.d, [&](int i) { return x[i]; });
            }
        }
        if (MAIN == kDelta && lane == 0) bulk_wait_le<0>();   // the results have been written
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0) {
        record_error(j.info, -KQ_ERR_TIMEOUT);
        // copies that this CTA sent to the other's barriers have had time to land
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 1000000ull) {
        }
    }
    cluster_barrier();   // neither CTA leaves while the other may still signal it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 2 * BN);
    }
}

// ---- few rows. The tiles above would take 256 of them whatever there are, and W would come in slower than memory can: here
// W's rows are the product's rows, 128 to a CTA, and N >= T tokens its columns. The results are taken through shared memory,
// so that a thread keeps the sums of one token from tile to tile. (8 rows of 128000 x 4096: 162 us, 6.5 TB/s; with the tiles
// above 254 us.)
constexpr int kThinThreads = 320;                // loads, products, 8 warps for the results
constexpr int kThinRows = 128, kThinMost = 128;  // rows of W of a tile, tokens
constexpr int kThinLd = kThinRows + 4;           // floats between tokens in shared memory
template <int N>
struct Thin {
    static constexpr int kStage = 2 * kBox + N * BK * 2;
    static constexpr int kOut = N * kThinLd * 4;
    static constexpr int kFit = (226 * 1024 - kOut - 1024) / kStage, kStages = kFit < 10 ? kFit : 10;
    static constexpr int kBoxRows = N <= 64 ? N : N / 2;   // of x
    static constexpr uint32_t kColumns = N == 32 ? 64 : N == 64 ? 128 : 256;   // two accumulators, a power of two
    static constexpr int kSmem = kStages * kStage + kOut + 1024;
};

template <int N>
__global__ void __launch_bounds__(kThinThreads, 1)
linear_thin_kernel(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw, const __grid_constant__ Job j) {
    using S = Thin<N>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    float* out = reinterpret_cast<float*>(smem + S::kStages * S::kStage);   // [N][kThinLd]
    __shared__ uint64_t full[S::kStages], empty[S::kStages], tfull[2], tempty[2], mma_done;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tfull[b], 1);
            mbar_init(&tempty[b], 8);
        }
        mbar_init(&mma_done, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_slot, S::kColumns);
        tmem_relinquish();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&mx);
        tma_prefetch_desc(&mw);
    }
    pdl_wait();
    pdl_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int tiles = static_cast<int>((j.w_main + kThinRows - 1) / kThinRows), slabs = static_cast<int>((j.d + BK - 1) / BK);

    if (warp == 0) {
        if (lane == 0) {
            int k = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                const int v = static_cast<int>(j.v_main) + t * kThinRows;
                for (int s = 0; s < slabs; ++s, ++k) {
                    const int st = k % S::kStages;
                    if (!held_wait(&empty[st], (static_cast<uint32_t>(k / S::kStages) & 1u) ^ 1u, &abort_flag)) {
                        ok = false;
                        break;
                    }
                    mbar_arrive_expect_tx(&full[st], S::kStage);
                    uint8_t* base = smem + st * S::kStage;
                    tma_load_2d(base, &mw, &full[st], s * BK, v);
                    tma_load_2d(base + kBox, &mw, &full[st], s * BK, v + 64);
#pragma unroll
                    for (int i = 0; i < N / S::kBoxRows; ++i)
                        tma_load_2d(base + 2 * kBox + i * S::kBoxRows * BK * 2, &mx, &full[st], s * BK, i * S::kBoxRows);
                }
            }
            for (int i = (k > S::kStages ? k - S::kStages : 0); i < k; ++i)   // whatever is under way has landed
                wait_quiet(&full[i % S::kStages], static_cast<uint32_t>(i / S::kStages) & 1u);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = idesc_bf16_mn_major(kThinRows, N) & ~(3u << 15);
            int k = 0, cc = 0;
            bool ok = true;
            for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
                for (int s0 = 0; s0 < slabs && ok; s0 += kDrainThin, ++cc) {
                    const int buf = cc & 1;
                    if (!held_wait(&tempty[buf], ((static_cast<uint32_t>(cc) >> 1) & 1u) ^ 1u, &abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const int s1 = min(slabs, s0 + kDrainThin);
                    for (int s = s0; s < s1; ++s, ++k) {
                        const int st = k % S::kStages;
                        if (!held_wait(&full[st], static_cast<uint32_t>(k / S::kStages) & 1u, &abort_flag)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        const uint32_t sa = smem_u32(smem + st * S::kStage), sb = sa + 2 * kBox;
#pragma unroll
                        for (int q = 0; q < BK / 16; ++q)
                            tc_mma_f16(tmem + buf * N, smem_desc_sw128(sa + q * 32, 16, 1024), smem_desc_sw128(sb + q * 32, 16, 1024), idesc,
                                       (s > s0 || q > 0) ? 1u : 0u);
                        tc_commit(&empty[st]);
                    }
                    if (ok) tc_commit(&tfull[buf]);
                }
            }
            tc_commit(&mma_done);
            wait_quiet(&mma_done, 0);
        }
    } else {
        // a thread takes half of the tokens of a row of W from tensor memory, then works on some rows of one token
        constexpr int kHalf = N / 2, kShare = N == 32 ? 8 : N == 64 ? 4 : 2, kPart = kThinRows / kShare;
        const int q = warp & 3, h = (warp - 2) >> 2, row = q * 32 + lane, id = threadIdx.x - 64;
        const int token = id / kShare, from = id % kShare * kPart;
        const bool mine = token < N && token < j.T;
        const int64_t y = mine ? j.target[token] : -1;
        Sums sums = {-INFINITY, 0.0f, 0.0f};
        int cc = 0;
        bool ok = true;
        for (int t = blockIdx.x; t < tiles && ok; t += gridDim.x) {
            float x[kHalf];
            for (int s0 = 0; s0 < slabs; s0 += kDrainThin, ++cc) {
                const int buf = cc & 1;
                ok = held_wait(&tfull[buf], (static_cast<uint32_t>(cc) >> 1) & 1u, &abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int p = 0; p < kHalf / 16; ++p) {
                    float v[16];
                    tmem_ld16(tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(buf * N + h * kHalf + p * 16), v);
                    tc_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[p * 16 + i] = s0 ? x[p * 16 + i] + v[i] : v[i];
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&tempty[buf]);
            }
            ok = named_all(ok);   // the others have read the last tile's, and none has given up
            if (!ok) break;
            const int64_t v0 = j.v_main + static_cast<int64_t>(t) * kThinRows;
            // past the vocabulary: cannot occur
#pragma unroll
            for (int i = 0; i < kHalf; ++i) out[(h * kHalf + i) * kThinLd + row] = v0 + row < j.V ? x[i] : -INFINITY;
            named_all(true);
            if (mine) {
                const float4* at = reinterpret_cast<const float4*>(out + token * kThinLd + from);
                float m = -INFINITY;
#pragma unroll 8
                for (int i = 0; i < kPart / 4; ++i) {
                    const float4 a = at[i];
                    m = max_nan(max_nan(m, max_nan(a.x, a.y)), max_nan(a.z, a.w));
                }
                const float ref = m == -INFINITY ? 0.0f : m;
                float z[4] = {0.0f, 0.0f, 0.0f, 0.0f}, s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
                for (int i = 0; i < kPart / 4; ++i) {
                    const float4 a = at[i];
                    const float w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float u = fmaxf((w[k] - ref) * kLog2e, kNone), e = ex2(u);
                        z[k] += e;
                        s[k] = fmaf(e, u, s[k]);
                    }
                }
                sums.join(m, (z[0] + z[1]) + (z[2] + z[3]), (s[0] + s[1]) + (s[2] + s[3]));
                const int64_t yr = y - v0 - from;
                if (y >= 0 && y < j.V && yr >= 0 && yr < kPart) j.zt[token] = out[token * kThinLd + from + yr];
            }
            __syncwarp();
        }
#pragma unroll
        for (int o = 1; o < kShare; o <<= 1)
            sums.join(__shfl_xor_sync(0xffffffffu, sums.m, o), __shfl_xor_sync(0xffffffffu, sums.z, o),
                      __shfl_xor_sync(0xffffffffu, sums.s, o));
        if (mine && from == 0 && KQ_IN_RANGE(blockIdx.x, j.parts))
            j.part[static_cast<int64_t>(token) * j.parts + blockIdx.x] = make_float4(sums.m, sums.z, sums.s, 0.0f);
    }
    tc_fence_before();
    __syncthreads();
    if (abort_flag && threadIdx.x == 0) record_error(j.info, -KQ_ERR_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, S::kColumns);
    }
}

// What D of a token needs, for n tokens by 256 threads.
__device__ __forceinline__ void fill_known(const Job& j, int n, int thread, float4* known, int* target) {
    for (int t = thread; t < n; t += 256) {
        const bool is = t < j.T;
        const int64_t y = is ? j.target[t] : -1;
        const bool scored = y >= 0 && y < j.V;
        const float lse = is ? j.lse[t] : -INFINITY;
        // a row of -infinity only, or none: p = 0 of every logit
        known[t] = make_float4(lse == -INFINITY ? INFINITY : lse, scored ? j.g_logp[t] : 0.0f, is && j.g_entropy ? j.g_entropy[t] : 0.0f,
                               is && j.g_entropy ? j.entropy[t] : 0.0f);
        target[t] = scored && lse != -INFINITY ? static_cast<int>(y) : -1;
    }
}

// ---- few rows, backwards. A CTA takes 128 rows of W at a time: their logits (the rows of W by N tokens), D, and the rows of gW:
// D, rounded to bf16, goes to shared memory as the operand of D x, 128 columns of gW at a time, and to `delta` (a row of N tokens
// for each row of W) for gx. One tile's products D x are issued between the next one's slabs, so that W's rows come in while gW's
// go out; both are bytes that nothing else moves (W twice with gx).
// Measured: 16 rows of 128000 x 4096 341 us for 2.1 GB; 96 rows of 128000 x 2048 190 us, 5.5 TB/s; 32 rows of that 173 us, and 253
// as two kernels, D and then its product. gx is left to the tiles above: with 64 columns of W and a share of its rows to a
// CTA, joined in a cluster, it took half as long again.
constexpr int kWide = 128;                       // columns of gW at a time
// Rows of W from which on gW comes in the same pass, half a tile for each SM: with fewer the tiles of a launch with gx share it out
// better (36 rows of d = 4064, both gradients: V = 8000 74 us in one pass and 62 apart, 16000 91 and 96, 32001 160 and 178; 96 rows
// of 1024: 33 and 32, 36 and 39, 63 and 63).
constexpr int64_t kFused = 10240;
template <int N>
struct ThinGrad {
    static constexpr int kBlocks = (N + 63) / 64;                       // of 64 tokens
    static constexpr int kBoxRows = Thin<N>::kBoxRows, kXBox = kBoxRows * 128, kXBoxes = N / kBoxRows;   // tokens of a box of x, bytes, boxes
    static constexpr int kStage = 2 * kBox + N * BK * 2, kColumnsOfX = 2 * kXBoxes * kXBox;   // a slab; kWide columns of x
    static constexpr int kD = kBlocks * 2 * kBox;                       // D of a tile
    static constexpr int kKnown = N * 20;
    static constexpr int kFit = (226 * 1024 - kD - 8 * kOutBox - kKnown - 1024) / kStage, kStages = kFit < 8 ? kFit : 8;
    static constexpr uint32_t kColumns = 512;                           // two accumulators of N and two of kWide
    static constexpr int kSmem = kStages * kStage + kD + 8 * kOutBox + kKnown + 1024;
    static_assert(kStage % 1024 == 0 && kStages >= 3 && kColumnsOfX <= kStage, "stages");
};

template <int N>
__global__ void __launch_bounds__(kThinThreads, 1)
linear_thin_grad_kernel(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw,
                        const __grid_constant__ CUtensorMap out_w, const __grid_constant__ Job j) {
    using S = ThinGrad<N>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    uint8_t* dop = smem + S::kStages * S::kStage;           // D as an operand: blocks of 64 tokens, 128-byte lines of a row of W
    uint8_t* boxes = dop + S::kD;
    float4* known = reinterpret_cast<float4*>(boxes + 8 * kOutBox);   // of each token: log-sum, the gradients, entropy
    int* target = reinterpret_cast<int*>(known + N);
    __shared__ uint64_t full[S::kStages], empty[S::kStages], zfull[2], zempty[2], gfull[2], gempty[2], dfull, mma_done;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&zfull[b], 1);
            mbar_init(&zempty[b], 8);
            mbar_init(&gfull[b], 1);
            mbar_init(&gempty[b], 8);
        }
        mbar_init(&dfull, 8);
        mbar_init(&mma_done, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_slot, S::kColumns);
        tmem_relinquish();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&mx);
        tma_prefetch_desc(&mw);
        tma_prefetch_desc(&out_w);
    }
    pdl_wait();
    pdl_launch_dependents();
    if (threadIdx.x >= 64) fill_known(j, N, threadIdx.x - 64, known, target);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int tiles = static_cast<int>((j.V + kThinRows - 1) / kThinRows), step = gridDim.x;
    const int mine = (tiles - static_cast<int>(blockIdx.x) + step - 1) / step;     // tiles of this CTA; the grid has no more CTAs than tiles
    const int slabs = j.d_slabs, turns = (slabs + 1) / 2;                          // a turn: kWide columns of gW, two slabs

    if (warp == 0) {
        if (lane == 0) {
            int k = 0;
            bool ok = true;
            auto room = [&](uint32_t bytes) {
                const int st = k % S::kStages;
                ok = ok && held_wait(&empty[st], (static_cast<uint32_t>(k / S::kStages) & 1u) ^ 1u, &abort_flag);
                if (ok) mbar_arrive_expect_tx(&full[st], bytes);
                return ok;
            };
            for (int r = 0; r <= mine && ok; ++r) {
                const int v = (static_cast<int>(blockIdx.x) + r * step) * kThinRows;
                for (int c = 0; c < turns && ok; ++c) {
                    if (r > 0 && j.gw) {
                        if (!room(S::kColumnsOfX)) break;
                        uint8_t* base = smem + k % S::kStages * S::kStage;
#pragma unroll
                        for (int i = 0; i < 2 * S::kXBoxes; ++i)
                            tma_load_2d(base + i * S::kXBox, &mx, &full[k % S::kStages], c * kWide + (i & 1) * 64, (i >> 1) * S::kBoxRows);
                        ++k;
                    }
                    for (int s = 2 * c; r < mine && s < min(2 * c + 2, slabs); ++s) {
                        if (!room(S::kStage)) break;
                        uint8_t* base = smem + k % S::kStages * S::kStage;
                        uint64_t* bar = &full[k % S::kStages];
                        tma_load_2d(base, &mw, bar, s * BK, v);
                        tma_load_2d(base + kBox, &mw, bar, s * BK, v + 64);
#pragma unroll
                        for (int i = 0; i < S::kXBoxes; ++i)
                            tma_load_2d(base + 2 * kBox + i * S::kXBox, &mx, bar, s * BK, i * S::kBoxRows);
                        ++k;
                    }
                }
            }
            for (int i = (k > S::kStages ? k - S::kStages : 0); i < k; ++i)   // whatever is under way has landed
                wait_quiet(&full[i % S::kStages], static_cast<uint32_t>(i / S::kStages) & 1u);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t z_idesc = idesc_bf16_mn_major(kThinRows, N) & ~(3u << 15);
            constexpr uint32_t g_idesc = idesc_bf16_mn_major(kThinRows, kWide) & ~(1u << 15);   // x by columns
            int k = 0, zc = 0, gc = 0;
            bool ok = true;
            auto landed = [&] {
                ok = ok && held_wait(&full[k % S::kStages], static_cast<uint32_t>(k / S::kStages) & 1u, &abort_flag);
                tc_fence_after();
                return ok;
            };
            auto drained = [&](uint64_t* bars, int count) {
                ok = ok && held_wait(&bars[count & 1], ((static_cast<uint32_t>(count) >> 1) & 1u) ^ 1u, &abort_flag);
                tc_fence_after();
                return ok;
            };
            for (int r = 0; r <= mine && ok; ++r) {
                if (r > 0 && j.gw) {   // D of the last tile is there
                    ok = held_wait(&dfull, static_cast<uint32_t>(r - 1) & 1u, &abort_flag);
                    tc_fence_after();
                }
                for (int c = 0; c < turns && ok; ++c) {
                    if (r > 0 && j.gw) {
                        if (!drained(gempty, gc) || !landed()) break;
                        const uint32_t sa = smem_u32(dop), sb = smem_u32(smem + k % S::kStages * S::kStage);
#pragma unroll
                        for (int q = 0; q < N / 16; ++q)
                            tc_mma_f16(tmem + 2 * N + (gc & 1) * kWide, smem_desc_sw128(sa + q / 4 * 2 * kBox + q % 4 * 32, 16, 1024),
                                       smem_desc_sw128(sb + 16 * q / S::kBoxRows * 2 * S::kXBox + 16 * q % S::kBoxRows * 128, S::kXBox, 1024),
                                       g_idesc, q > 0 ? 1u : 0u);
                        tc_commit(&empty[k % S::kStages]);
                        tc_commit(&gfull[gc & 1]);
                        ++k, ++gc;
                    }
                    for (int s = 2 * c; r < mine && s < min(2 * c + 2, slabs); ++s) {
                        if (s % kDrainThin == 0 && !drained(zempty, zc)) break;
                        if (!landed()) break;
                        const uint32_t sa = smem_u32(smem + k % S::kStages * S::kStage), sb = sa + 2 * kBox;
#pragma unroll
                        for (int q = 0; q < BK / 16; ++q)
                            tc_mma_f16(tmem + (zc & 1) * N, smem_desc_sw128(sa + q * 32, 16, 1024), smem_desc_sw128(sb + q * 32, 16, 1024),
                                       z_idesc, (s % kDrainThin > 0 || q > 0) ? 1u : 0u);
                        tc_commit(&empty[k % S::kStages]);
                        ++k;
                        if (s % kDrainThin == kDrainThin - 1 || s == slabs - 1) {
                            tc_commit(&zfull[zc & 1]);
                            ++zc;
                        }
                    }
                }
            }
            tc_commit(&mma_done);
            wait_quiet(&mma_done, 0);
        }
    } else {
        constexpr int kHalf = N / 2;
        const int q = warp & 3, h = (warp - 2) >> 2, row = q * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(q * 32) << 16);
        uint8_t* box = boxes + (warp - 2) * kOutBox;
        int zc = 0, gc = 0;
        bool ok = true;
        auto filled = [&](uint64_t* bars, int count) {
            const bool is = held_wait(&bars[count & 1], (static_cast<uint32_t>(count) >> 1) & 1u, &abort_flag);
            ok = __all_sync(0xffffffffu, is);
            tc_fence_after();
            return ok;
        };
        auto drained = [&](uint64_t* bar) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        for (int r = 0; r <= mine && ok; ++r) {
            const int tile = static_cast<int>(blockIdx.x) + r * step;
            float x[kHalf];
            for (int c = 0; c < turns; ++c) {
                if (r > 0 && j.gw) {
                    if (!filled(gfull, gc)) break;
                    const uint32_t at = lanes + static_cast<uint32_t>(2 * N + (gc & 1) * kWide + h * 64);
                    float y[32];
                    put_begin();
                    tmem_ld32(at, y);
                    tc_wait_ld();
                    put_part<0, 4>(box, [&](int i) { return y[i]; });
                    tmem_ld32(at + 32, y);
                    tc_wait_ld();
                    drained(&gempty[gc & 1]);
                    ++gc;
                    put_part<4, 8>(box, [&](int i) { return y[i - 32]; });
                    put_end(box, &out_w, static_cast<int64_t>(tile - step) * kThinRows + q * 32, j.V, c * kWide + h * 64, j.d);
                }
                const int s = min(2 * c + 2, slabs);   // slabs that this turn ends with
                if (r < mine && (s % kDrainThin == 0 || s == slabs)) {
                    if (!filled(zfull, zc)) break;
#pragma unroll
                    for (int p = 0; p < kHalf / 16; ++p) {
                        float v[16];
                        tmem_ld16(lanes + static_cast<uint32_t>((zc & 1) * N + h * kHalf + p * 16), v);
                        tc_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[p * 16 + i] = s > kDrainThin ? x[p * 16 + i] + v[i] : v[i];
                    }
                    drained(&zempty[zc & 1]);
                    ++zc;
                }
            }
            if (!ok || r == mine) break;
            // D; the last tile's products with it have been read out, so its operand may be written over
            const int64_t v = static_cast<int64_t>(tile) * kThinRows + row;
            __nv_bfloat16* dst = j.delta + v * N + h * kHalf;
            const bool put = j.delta && KQ_IN_RANGE(v, j.ld_delta);
            // whether a target of this warp's tokens lies in the tile, which is rare
            bool hit = false;
#pragma unroll
            for (int t = 0; t < kHalf; t += 32)
                if (t + lane < kHalf) hit |= static_cast<unsigned>(target[h * kHalf + t + lane] - tile * kThinRows) < kThinRows;
            hit = __any_sync(0xffffffffu, hit);
#pragma unroll
            for (int c = 0; c < kHalf / 8; ++c) {
                const int at = h * kHalf + 8 * c;
                float d[8];
                if (j.g_entropy) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 a = known[at + e];
                        d[e] = delta_of(x[8 * c + e], a.x, a.y, a.z, a.w);
                    }
                } else {   // the same without the entropy's part
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 a = *reinterpret_cast<const float2*>(known + at + e);
                        d[e] = -a.y * ex2((x[8 * c + e] - a.x) * kLog2e);
                    }
                }
                if (hit) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (target[at + e] == v) d[e] += known[at + e].y;
                }
                uint4 w = make_uint4(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4], d[5]), pack_bf16(d[6], d[7]));
                if (v >= j.V) w = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(dop + at / 64 * 2 * kBox + row * 128 + ((at % 64 / 8) ^ (row & 7)) * 16) = w;
                if (put) *reinterpret_cast<uint4*>(dst + 8 * c) = w;
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&dfull);
        }
        if (lane == 0) bulk_wait_le<0>();   // the results have been written
    }
    tc_fence_before();
    __syncthreads();
    if (abort_flag && threadIdx.x == 0) record_error(j.info, -KQ_ERR_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, S::kColumns);
    }
}

// ---- few rows and a small vocabulary: fewer tiles of W than SMs. A cluster takes a tile, its CTAs a share of d each; a CTA adds up
// the shares of its part of the tile's rows, in their order, from what the others have put into its shared memory.
// A CTA alone takes 0.28 us for each slab of a tile, whatever the other SMs do, so that a long d with few tiles is bound by one CTA:
// 9 rows of 1900 x 6304 took 31 us and take 10.7 (24 MB, 4 us at the copy's rate), with both gradients 60 and 28.
template <int N>
struct Split {
    static constexpr int kStage = Thin<N>::kStage, kBoxRows = Thin<N>::kBoxRows, kMail = N * (kThinRows + 8) * 4;
    static constexpr uint32_t kColumns = Thin<N>::kColumns;
    static constexpr int kFit = (226 * 1024 - kMail - N * 20 - 1024) / kStage, kStages = kFit < 10 ? kFit : 10;
    static constexpr int kSmem = kStages * kStage + kMail + N * 20 + 1024;
};

template <int MAIN, int N>
__global__ void __launch_bounds__(kThinThreads, 1)
linear_split_kernel(const __grid_constant__ CUtensorMap mx, const __grid_constant__ CUtensorMap mw, const __grid_constant__ Job j) {
    using S = Split<N>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    float* mail = reinterpret_cast<float*>(smem + S::kStages * S::kStage);   // [shares][N][rows of this CTA and one]
    float4* known = reinterpret_cast<float4*>(mail + N * (kThinRows + 8));    // of each token: log-sum, the gradients, entropy
    int* target = reinterpret_cast<int*>(known + N);
    __shared__ uint64_t full[S::kStages], empty[S::kStages], tfull[2], tempty[2], mma_done;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&tfull[b], 1);
            mbar_init(&tempty[b], 8);
        }
        mbar_init(&mma_done, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(&tmem_slot, S::kColumns);
        tmem_relinquish();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&mx);
        tma_prefetch_desc(&mw);
    }
    pdl_wait();
    pdl_launch_dependents();
    if (MAIN == kDelta && threadIdx.x >= 64) fill_known(j, N, threadIdx.x - 64, known, target);
    tc_fence_before();
    __syncthreads();
    cluster_barrier();   // every CTA's mail is there
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int shares = gridDim.x, share = blockIdx.x, tile = blockIdx.y, rows = kThinRows / shares;
    const int each = (j.d_slabs + shares - 1) / shares, first = share * each, slabs = max(0, min(each, j.d_slabs - first));

    if (warp == 0) {
        if (lane == 0) {
            int k = 0;
            for (; k < slabs; ++k) {
                const int st = k % S::kStages, x = (first + k) * BK;
                if (!held_wait(&empty[st], (static_cast<uint32_t>(k / S::kStages) & 1u) ^ 1u, &abort_flag)) break;
                mbar_arrive_expect_tx(&full[st], S::kStage);
                uint8_t* base = smem + st * S::kStage;
                tma_load_2d(base, &mw, &full[st], x, tile * kThinRows);
                tma_load_2d(base + kBox, &mw, &full[st], x, tile * kThinRows + 64);
#pragma unroll
                for (int i = 0; i < N / S::kBoxRows; ++i)
                    tma_load_2d(base + 2 * kBox + i * S::kBoxRows * BK * 2, &mx, &full[st], x, i * S::kBoxRows);
            }
            for (int i = (k > S::kStages ? k - S::kStages : 0); i < k; ++i)   // whatever is under way has landed
                wait_quiet(&full[i % S::kStages], static_cast<uint32_t>(i / S::kStages) & 1u);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t idesc = idesc_bf16_mn_major(kThinRows, N) & ~(3u << 15);
            int k = 0, cc = 0;
            bool ok = true;
            for (int s0 = 0; s0 < slabs && ok; s0 += kDrainThin, ++cc) {
                const int buf = cc & 1;
                if (!held_wait(&tempty[buf], ((static_cast<uint32_t>(cc) >> 1) & 1u) ^ 1u, &abort_flag)) break;
                tc_fence_after();
                for (const int s1 = min(slabs, s0 + kDrainThin); k < s1; ++k) {
                    const int st = k % S::kStages;
                    ok = held_wait(&full[st], static_cast<uint32_t>(k / S::kStages) & 1u, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = smem_u32(smem + st * S::kStage), sb = sa + 2 * kBox;
#pragma unroll
                    for (int q = 0; q < BK / 16; ++q)
                        tc_mma_f16(tmem + buf * N, smem_desc_sw128(sa + q * 32, 16, 1024), smem_desc_sw128(sb + q * 32, 16, 1024), idesc,
                                   (k > s0 || q > 0) ? 1u : 0u);
                    tc_commit(&empty[st]);
                }
                if (ok) tc_commit(&tfull[buf]);
            }
            tc_commit(&mma_done);
            wait_quiet(&mma_done, 0);
        }
    } else {
        constexpr int kHalf = N / 2;
        const int q = warp & 3, h = (warp - 2) >> 2, row = q * 32 + lane;
        float x[kHalf];
#pragma unroll
        for (int i = 0; i < kHalf; ++i) x[i] = 0.0f;
        for (int s0 = 0, cc = 0; s0 < slabs; s0 += kDrainThin, ++cc) {
            const int buf = cc & 1;
            const bool is = held_wait(&tfull[buf], (static_cast<uint32_t>(cc) >> 1) & 1u, &abort_flag);
            if (!__all_sync(0xffffffffu, is)) break;
            tc_fence_after();
#pragma unroll
            for (int p = 0; p < kHalf / 16; ++p) {
                float v[16];
                tmem_ld16(tmem + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(buf * N + h * kHalf + p * 16), v);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) x[p * 16 + i] += v[i];
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tempty[buf]);
        }
        // to the CTA that has this row of W
        const int owner = row / rows;
        const uint32_t at = mapa_shared(smem_u32(mail + (share * N + h * kHalf) * (rows + 1) + row % rows), owner);
#pragma unroll
        for (int i = 0; i < kHalf; ++i)
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + static_cast<uint32_t>(i * (rows + 1)) * 4), "f"(x[i]) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();
    const int64_t v0 = static_cast<int64_t>(tile) * kThinRows + share * rows;
    if (threadIdx.x >= 64) {
        const int id = threadIdx.x - 64, pitch = rows + 1;
        // the logits, in the place of the first share's; past the vocabulary: cannot occur
        for (int i = id; i < j.T * rows; i += 256) {
            const int token = i / rows, row = i - token * rows;
            float z = 0.0f;
            for (int o = 0; o < shares; ++o) z += mail[(o * N + token) * pitch + row];
            mail[token * pitch + row] = v0 + row < j.V ? z : -INFINITY;
        }
        named_all(true);
        if (MAIN == kScore) {
            constexpr int kShare = N == 32 ? 8 : N == 64 ? 4 : 2;   // threads of a token, which take its rows in turn
            const int token = id / kShare, from = id % kShare;
            const bool mine = token < N && token < j.T;
            Sums sums = {-INFINITY, 0.0f, 0.0f};
            if (mine) {
                const int64_t y = j.target[token] - v0;
                const float* z = mail + token * pitch;
                float m = -INFINITY;
                for (int i = from; i < rows; i += kShare) {
                    m = max_nan(m, z[i]);
                    if (y == i && v0 + i < j.V) j.zt[token] = z[i];
                }
                sums.m = m;
                const float ref = m == -INFINITY ? 0.0f : m;
                for (int i = from; i < rows; i += kShare) {
                    const float u = fmaxf((z[i] - ref) * kLog2e, kNone), e = ex2(u);
                    sums.z += e;
                    sums.s = fmaf(e, u, sums.s);
                }
            }
            __syncwarp();
#pragma unroll
            for (int o = 1; o < kShare; o <<= 1)
                sums.join(__shfl_xor_sync(0xffffffffu, sums.m, o), __shfl_xor_sync(0xffffffffu, sums.z, o),
                          __shfl_xor_sync(0xffffffffu, sums.s, o));
            if (mine && from == 0 && KQ_IN_RANGE(tile * shares + share, j.parts))
                j.part[static_cast<int64_t>(token) * j.parts + tile * shares + share] = make_float4(sums.m, sums.z, sums.s, 0.0f);
        } else {
            for (int i = id; i < rows * (N / 8); i += 256) {
                const int t0 = i / rows * 8, row = i - i / rows * rows;
                const int64_t v = v0 + row;
                float d[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float4 a = known[t0 + e];
                    d[e] = t0 + e < j.T && v < j.V ? delta_of(mail[(t0 + e) * pitch + row], a.x, a.y, a.z, a.w) : 0.0f;
                    if (target[t0 + e] == v) d[e] += a.y;
                }
                if (KQ_IN_RANGE(v, j.ld_delta))
                    *reinterpret_cast<uint4*>(j.delta + v * N + t0) =
                        make_uint4(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4], d[5]), pack_bf16(d[6], d[7]));
            }
        }
    }
    if (abort_flag && threadIdx.x == 0) record_error(j.info, -KQ_ERR_TIMEOUT);
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, S::kColumns);
    }
}

// Joins the parts of a row: a block to a row.
__global__ void __launch_bounds__(128) linear_join_kernel(const Job j, float* __restrict__ logp, float* __restrict__ entropy,
                                                          float* __restrict__ lse) {
    __shared__ float sm[4], sz[4], ss[4];
    const int64_t row = blockIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    const float4* p = j.part + row * j.parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums a = {-INFINITY, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < j.parts; i += 128) {
        const float4 v = p[i];
        a.join(v.x, v.y, v.z);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        a.join(__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.z, o), __shfl_xor_sync(0xffffffffu, a.s, o));
    if (lane == 0) sm[warp] = a.m, sz[warp] = a.z, ss[warp] = a.s;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 4; ++w) a.join(sm[w], sz[w], ss[w]);
    const float M = a.m, Z = a.z, S = a.s;
    const int64_t y = j.target[row];
    const bool none = M == -INFINITY;
    const float lz = log2f(Z), ln = lz * kLn2;
    if (y >= j.V) record_error(j.info, -KQ_ERR_INVALID_ARG);
    float lp = 0.0f;
    if (y >= j.V) lp = NAN;
    else if (y >= 0) lp = none ? -INFINITY : j.zt[row] - M - ln;
    logp[row] = lp > 0.0f ? 0.0f : lp;
    if (entropy) entropy[row] = none ? 0.0f : (lz - S / Z) * kLn2;
    if (lse) lse[row] = none ? -INFINITY : M + ln;
}

// gx = the sum of the splits, in order.
__global__ void __launch_bounds__(64) linear_gx_kernel(const float* __restrict__ sum, int splits, int64_t T, int64_t d,
                                                        __nv_bfloat16* __restrict__ gx, int64_t ld) {
    const int64_t each = T * d, per_row = d / 4;
    pdl_wait();
    pdl_launch_dependents();
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < T * per_row;
         i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int64_t row = i / per_row, col = (i - row * per_row) * 4;
        float x[4] = {};
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            const float4 a = *reinterpret_cast<const float4*>(sum + s * each + row * d + col);
            x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w;
        }
        if (KQ_IN_RANGE(row * ld + col + 3, (T - 1) * ld + d))
            *reinterpret_cast<uint2*>(gx + row * ld + col) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    }
}
// Targets past the vocabulary are reported; the gradient's tiles leave them out.
__global__ void linear_targets_kernel(const int64_t* __restrict__ target, int64_t T, int64_t V, int* info) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < T; i += static_cast<int64_t>(gridDim.x) * blockDim.x)
        if (target[i] >= V) record_error(info, -KQ_ERR_INVALID_ARG);
}

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Boxes of 64 columns and box_rows rows of a row-major bf16 matrix, 128-byte swizzle, zeros outside.
kq_status make_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t ld, const char* who, int box_rows = 64) {
    static std::atomic<EncodeTiledFn> fn{nullptr};
    EncodeTiledFn enc = fn.load();
    if (!enc) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            set_error("%s: cuTensorMapEncodeTiled is unavailable", who);
            return KQ_ERR_CUDA;
        }
        enc = reinterpret_cast<EncodeTiledFn>(p);
        fn.store(enc);
    }
    std::memset(m, 0, sizeof(*m));
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ld) * 2};
    const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)}, one[2] = {1, 1};
    const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, one,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("%s: cuTensorMapEncodeTiled failed (%d)", who, static_cast<int>(r));
        return KQ_ERR_CUDA;
    }
    return KQ_OK;
}

// The matrices of a launch: x, W, D that is read; D, gx and gw that are written.
struct Maps {
    CUtensorMap x, w, d, out_d, out_x, out_w;
};
int max_clusters() {
    static std::atomic<int> kept[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return num_sms() / 2;
    if (const int c = kept[dev].load()) return c;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(num_sms() / 2 * 2));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    int c = 0;
    if (cudaOccupancyMaxActiveClusters(&c, linear_tile_kernel<kScore>, &cfg) != cudaSuccess || c < 1) c = num_sms() / 2;
    kept[dev].store(c);
    return c;
}

// The pairs' runs of the logits' tiles: as many to each as bring it up to a common level of work, counted in slabs.
void even_out(Job& j, int pairs) {
    const int deal = j.t_gx + j.t_gw, main = j.tiles - deal;
    const int64_t cost = j.d_slabs + kTileCost;
    int64_t load[kMostPairs] = {}, all = main * cost;
    for (int t = 0, rd = 0; t < deal; t += pairs, ++rd)
        for (int p = 0; p < pairs; ++p) {
            const int at = round_tile(rd, p, pairs);
            if (at >= deal) continue;
            const int64_t slabs = at >= j.t_gx ? j.row_slabs
                                               : std::min(j.split_slabs, j.prod_slabs - at / (j.m_prod * j.n_d) * j.split_slabs);
            load[p] += slabs + kTileCost;
            all += slabs + kTileCost;
        }
    // the lowest level that takes them all, within a tile of the mean or of the fullest pair
    int64_t low = all / pairs, high = low + cost;
    for (int p = 0; p < pairs; ++p) high = std::max(high, load[p] + cost);
    auto room = [&](int64_t level, int p) { return level > load[p] ? (level - load[p]) / cost : 0; };
    while (low < high) {
        const int64_t mid = (low + high) / 2;
        int64_t sum = 0;
        for (int p = 0; p < pairs; ++p) sum += room(mid, p);
        if (sum >= main) high = mid;
        else low = mid + 1;
    }
    int64_t at = 0;
    for (int p = 0; p < pairs; ++p) {
        j.first_main[p] = static_cast<int32_t>(at);
        at = std::min<int64_t>(main, at + room(low, p));
    }
    j.first_main[pairs] = static_cast<int32_t>(main);
}

template <int MAIN>
kq_status run_tiles(const Maps& m, Job& j, cudaStream_t stream) {
    if (j.tiles == 0) return KQ_OK;
    int pairs = std::min(j.tiles, max_clusters());
    if (j.t_gx + j.t_gw) {
        pairs = std::min(pairs, kMostPairs);
        even_out(j, pairs);
    }
    KQ_CUDA(launch_after(linear_tile_kernel<MAIN>, dim3(static_cast<unsigned>(2 * pairs)), dim3(kThreads), kSmem, stream, m.x, m.w, m.d,
                         m.out_d, m.out_x, m.out_w, j));
    count_launch();
    return KQ_OK;
}
template <typename K, typename... Args>
kq_status run_thin_kernel(K kernel, int smem, std::atomic<uint64_t>& done, int64_t blocks, cudaStream_t stream, const Args&... args) {
    KQ_TRY(once_per_device(done, [&] {
        KQ_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        return KQ_OK;
    }));
    KQ_CUDA(launch_after(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThinThreads), smem, stream, args...));
    count_launch();
    return KQ_OK;
}
int64_t thin_blocks(int64_t V) { return std::min<int64_t>(cdiv(V, kThinRows), num_sms()); }
// Tokens that a product has room for, and rows of a box of x.
int thin_tokens(int64_t T) { return T <= 32 ? 32 : T <= 64 ? 64 : T <= 96 ? 96 : 128; }
int thin_box_rows(int n) { return n <= 64 ? n : n / 2; }

// The shares of d that a tile of W is cut into: as many as there are SMs for (152 SMs hold 76 clusters of 2 such CTAs, 36 of 4 or 15
// of 8; with one cluster more, 38 of 4, 120 rows of 4864 x 2048 took 25 us instead of 16). Sums between CTAs cost as much as some
// slabs, more for more tokens, so a share has to leave that many to the others. Scores, whole and in shares: 12 x 2583 x 3040 18 and 10
// us, 100 x 3900 x 4096 25 and 16, 30 x 8000 x 2048 14 and 13, but 60 x 8000 x 2048 14.8 and 15.1, 100 x 8000 x 2048 16 and 19, 20 x
// 1000 x 512 7.0 and 8.6. D's kernel gains sooner (all of a gradient, 100 x 8000 x 2048: 46 and 42 us; 20 x 1000 x 512: 13.8 and 14.4).
int split_shares(const Job& j, bool score) {
    const int64_t tiles = cdiv(j.V, kThinRows);
    int shares = 1;
    while (shares < 8 && tiles * shares * 2 <= num_sms() - 8 * shares && j.d_slabs >= 8 * shares) shares *= 2;
    return j.d_slabs - cdiv(j.d_slabs, shares) > (score ? thin_tokens(j.T) / 4 : 4) ? shares : 1;
}
template <int MAIN, int N>
kq_status run_split(const Maps& m, Job& j, int shares, cudaStream_t stream) {
    static std::atomic<uint64_t> done{0};
    KQ_TRY(once_per_device(done, [] {
        KQ_CUDA(cudaFuncSetAttribute(linear_split_kernel<MAIN, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, Split<N>::kSmem));
        return KQ_OK;
    }));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(shares), static_cast<unsigned>(cdiv(j.V, kThinRows)));
    cfg.blockDim = dim3(kThinThreads);
    cfg.dynamicSmemBytes = Split<N>::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = static_cast<unsigned>(shares);
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    j.parts = static_cast<int32_t>(cdiv(j.V, kThinRows) * shares);
    KQ_CUDA(cudaLaunchKernelEx(&cfg, linear_split_kernel<MAIN, N>, m.x, m.w, static_cast<const Job>(j)));
    count_launch();
    return KQ_OK;
}

template <int N>
kq_status run_thin_of(const Maps& m, Job& j, cudaStream_t stream) {
    static std::atomic<uint64_t> done{0};
    if (const int shares = split_shares(j, true); shares > 1) return run_split<kScore, N>(m, j, shares, stream);
    j.parts = static_cast<int32_t>(thin_blocks(j.V));
    return run_thin_kernel(linear_thin_kernel<N>, Thin<N>::kSmem, done, j.parts, stream, m.x, m.w, j);
}
kq_status run_thin(const Maps& m, Job& j, cudaStream_t stream) {
    switch (thin_tokens(j.T)) {
        case 32: return run_thin_of<32>(m, j, stream);
        case 64: return run_thin_of<64>(m, j, stream);
        case 96: return run_thin_of<96>(m, j, stream);
        default: return run_thin_of<128>(m, j, stream);
    }
}
template <int N>
kq_status run_thin_grad_of(const Maps& m, Job& j, cudaStream_t stream) {
    static std::atomic<uint64_t> done{0};
    if (const int shares = split_shares(j, false); shares > 1 && !j.gw) return run_split<kDelta, N>(m, j, shares, stream);
    return run_thin_kernel(linear_thin_grad_kernel<N>, ThinGrad<N>::kSmem, done, thin_blocks(j.V), stream, m.x, m.w, m.out_w, j);
}
kq_status run_thin_grad(const Maps& m, Job& j, cudaStream_t stream) {
    switch (thin_tokens(j.T)) {
        case 32: return run_thin_grad_of<32>(m, j, stream);
        case 64: return run_thin_grad_of<64>(m, j, stream);
        case 96: return run_thin_grad_of<96>(m, j, stream);
        default: return run_thin_grad_of<128>(m, j, stream);
    }
}
kq_status set_up() {
    static std::atomic<uint64_t> done{0};
    return once_per_device(done, [] {
        KQ_CUDA(cudaFuncSetAttribute(linear_tile_kernel<kScore>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
        KQ_CUDA(cudaFuncSetAttribute(linear_tile_kernel<kDelta>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
        return KQ_OK;
    });
}

// How the gradient is cut; from the sizes alone, so that the workspace's size is the same on every device.
struct Cut {
    int64_t piece;        // columns
    int64_t pieces;
    int32_t splits, split_slabs;
    size_t delta, sum;    // bytes of one of the two D, of gx so far
};
Cut cut_of(int64_t T, int64_t V, int64_t d) {
    Cut c;
    // few rows have D of the whole vocabulary, at most 2^27 values, by rows of W
    const int64_t columns = T <= kThinMost ? V : std::max(kLeastPiece, kPiece / T / BN * BN);
    c.piece = std::min(cdiv(columns, BN) * BN, cdiv(V, BN) * BN);
    c.pieces = cdiv(V, c.piece);
    const int64_t tiles = cdiv(T, BM) * cdiv(d, BN), slabs = cdiv(std::min(c.piece, V), BK);   // of the first piece
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(76 / tiles, slabs / 4));
    c.split_slabs = static_cast<int32_t>(cdiv(slabs, splits));
    c.splits = static_cast<int32_t>(cdiv(slabs, c.split_slabs));
    c.delta = static_cast<size_t>(T <= kThinMost ? thin_tokens(T) : T) * c.piece * 2;
    c.sum = c.pieces * c.splits > 1 ? static_cast<size_t>(c.splits) * T * d * sizeof(float) : 0;
    return c;
}
size_t al256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }
// Rows that scoring has room for at once, whole bands: their parts, 16 bytes for 64 logits, are joined before the next rows come, so
// that the workspace does not grow with the rows. At 2^29 logits or more a time that costs 1 to 2 % (16384 rows of 131072 x 512 by 8192
// 1.45 and 1.46 ms, of 131072 x 64 1.14 and 1.16; 65536 of 128000 x 2048 19.5 and 19.5).
int64_t score_room(int64_t V) {
    constexpr int64_t band = kBand * BM;
    return std::max(band, kMostParts / cdiv(V, 64) / band * band);
}
// Rows of each time: as many times as the room asks for, evenly, as a time of a few rows reads W for them alone.
int64_t score_rows(int64_t T, int64_t V) {
    const int64_t times = cdiv(T, score_room(V));
    return times == 1 ? T : cdiv(cdiv(T, times), BM) * BM;
}
// Parts of a row's sums: 64 columns of a tile, or the rows of W that a CTA has of one of few tiles.
int64_t most_parts(int64_t T, int64_t V) {
    return T <= kThinMost ? std::max(cdiv(V, 64), 8 * std::min<int64_t>(cdiv(V, kThinRows), 128)) : cdiv(V, 64);
}

kq_status check(const char* who, const uint16_t* x, int64_t T, int64_t d, int64_t ldx, const uint16_t* w, int64_t V, int64_t ldw,
                const int64_t* target) {
    if (V > KQ_LOGPROBS_MAX_V || d > 65536 || d % 8) {
        set_error("%s: V must be at most %d, d a multiple of 8 up to 65536", who, KQ_LOGPROBS_MAX_V);
        return KQ_ERR_UNSUPPORTED;
    }
    if (T < 0 || T > KQ_LINEAR_MAX_T || V < 1 || d < 1 || !w || ldw < d || ldx < d || ((ldx | ldw) & 7) || (T > 0 && (!x || !target)) ||
        ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(w)) & 15u)) {
        set_error("%s: x, w and target must not be NULL, x and w 16-byte aligned with row strides of at least d in multiples of 8, "
                  "0 <= T <= %d, V >= 1", who, KQ_LINEAR_MAX_T);
        return KQ_ERR_INVALID_ARG;
    }
    return KQ_OK;
}

}  // namespace

KQ_DEBUG_UNIT(linear_logprob)
}  // namespace kq

using namespace kq;

extern "C" size_t kq_linear_logprobs_workspace(int64_t T, int64_t V, int64_t d) {
    if (T < 1 || V < 1 || d < 1) return 0;
    const int64_t rows = std::min(T, score_room(V));
    return al256(static_cast<size_t>(rows) * most_parts(T, V) * sizeof(float4)) + al256(rows * sizeof(float));
}

extern "C" kq_status kq_linear_logprobs(const uint16_t* x, int64_t T, int64_t d, int64_t ldx, const uint16_t* w, int64_t V, int64_t ldw,
                                        const int64_t* target, float* logp, float* entropy, float* lse, int* info, void* ws,
                                        size_t ws_bytes, kq_stream_t stream_) {
    const char* who = "kq_linear_logprobs";
    KQ_TRY(check(who, x, T, d, ldx, w, V, ldw, target));
    if (T == 0) return KQ_OK;
    if (!logp) {
        set_error("%s: logp must not be NULL", who);
        return KQ_ERR_INVALID_ARG;
    }
    const size_t need = kq_linear_logprobs_workspace(T, V, d);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("%s: workspace must be 256-byte aligned and hold %zu bytes", who, need);
        return KQ_ERR_WORKSPACE;
    }
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    KQ_TRY(set_up());
    Maps m;
    KQ_TRY(make_map(&m.w, w, V, d, ldw, who));
    m.d = m.out_d = m.out_x = m.out_w = m.w;   // not used
    const bool thin = T <= kThinMost;
    const int64_t rows = score_rows(T, V), room = std::min(T, score_room(V));
    Job j = {};
    j.V = V, j.d = d;
    j.part = static_cast<float4*>(ws);
    j.zt = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + al256(static_cast<size_t>(room) * most_parts(T, V) * sizeof(float4)));
    j.n_main = static_cast<int32_t>(cdiv(V, BN));
    j.w_main = V;
    j.d_slabs = static_cast<int32_t>(cdiv(d, BK));
    j.info = info;
    for (int64_t r = 0; r < T; r += rows) {
        j.T = std::min(rows, T - r);
        KQ_TRY(make_map(&m.x, x + r * ldx, j.T, d, ldx, who, thin ? thin_box_rows(thin_tokens(T)) : 64));
        j.target = target + r;
        j.parts = static_cast<int32_t>(cdiv(V, 64));
        j.m_main = static_cast<int32_t>(cdiv(j.T, BM));
        j.tiles = j.m_main * j.n_main;
        KQ_TRY(thin ? run_thin(m, j, stream) : run_tiles<kScore>(m, j, stream));
        KQ_CUDA(launch_after(linear_join_kernel, dim3(static_cast<unsigned>(j.T)), dim3(128), 0, stream, j, logp + r,
                             entropy ? entropy + r : nullptr, lse ? lse + r : nullptr));
        count_launch();
    }
    return KQ_OK;
}

extern "C" size_t kq_linear_logprobs_grad_workspace(int64_t T, int64_t V, int64_t d) {
    if (T < 1 || V < 1 || d < 1) return 0;
    const Cut c = cut_of(T, V, d);
    return al256(c.delta) * (c.pieces > 1 ? 2 : 1) + al256(c.sum);
}

extern "C" kq_status kq_linear_logprobs_grad(const uint16_t* x, int64_t T, int64_t d, int64_t ldx, const uint16_t* w, int64_t V,
                                             int64_t ldw, const int64_t* target, const float* lse, const float* entropy,
                                             const float* g_logp, const float* g_entropy, uint16_t* gx, int64_t ldgx, uint16_t* gw,
                                             int64_t ldgw, int* info, void* ws, size_t ws_bytes, kq_stream_t stream_) {
    const char* who = "kq_linear_logprobs_grad";
    KQ_TRY(check(who, x, T, d, ldx, w, V, ldw, target));
    if ((T > 0 && (!lse || !g_logp || (g_entropy && !entropy))) || (!gx && !gw) || (gx && (ldgx < d || (ldgx & 7))) ||
        (gw && (ldgw < d || (ldgw & 7))) || ((reinterpret_cast<uintptr_t>(gx) | reinterpret_cast<uintptr_t>(gw)) & 15u)) {
        set_error("%s: lse, g_logp (and entropy with g_entropy) and gx or gw must not be NULL, gx and gw 16-byte aligned with row "
                  "strides of at least d in multiples of 8", who);
        return KQ_ERR_INVALID_ARG;
    }
    // later pieces read x and W again
    if (T > 0 && ((gx && (gx == x || gx == w)) || (gw && (gw == w || gw == x)) || (gx && gx == gw))) {
        set_error("%s: gx and gw must not be x, w or each other", who);
        return KQ_ERR_INVALID_ARG;
    }
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    if (T == 0) {
        if (gw) KQ_CUDA(cudaMemset2DAsync(gw, ldgw * 2, 0, d * 2, V, stream));
        return KQ_OK;
    }
    const size_t need = kq_linear_logprobs_grad_workspace(T, V, d);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("%s: workspace must be 256-byte aligned and hold %zu bytes", who, need);
        return KQ_ERR_WORKSPACE;
    }
    KQ_TRY(set_up());
    const Cut c = cut_of(T, V, d);
    uint8_t* at = static_cast<uint8_t*>(ws);
    __nv_bfloat16* delta[2] = {reinterpret_cast<__nv_bfloat16*>(at),
                               reinterpret_cast<__nv_bfloat16*>(at + (c.pieces > 1 ? al256(c.delta) : 0))};
    Maps m;
    CUtensorMap read[2], write[2];
    const bool thin = T <= kThinMost;
    const int n = thin_tokens(T);
    KQ_TRY(make_map(&m.x, x, T, d, ldx, who));
    KQ_TRY(make_map(&m.w, w, V, d, ldw, who));
    m.out_x = m.out_w = m.w;
    if (gx) KQ_TRY(make_map(&m.out_x, gx, T, d, ldgx, who, 32));
    if (gw) KQ_TRY(make_map(&m.out_w, gw, V, d, ldgw, who, 32));
    for (int i = 0; i < 2; ++i) {
        if (thin) KQ_TRY(make_map(&read[i], delta[i], V, n, n, who));
        else KQ_TRY(make_map(&read[i], delta[i], T, c.piece, c.piece, who));
        write[i] = read[i];
        if (!thin) KQ_TRY(make_map(&write[i], delta[i], T, c.piece, c.piece, who, 32));
    }
    if (info) {
        linear_targets_kernel<<<static_cast<unsigned>(std::min<int64_t>(cdiv(T, 256), 1024)), 256, 0, stream>>>(target, T, V, info);
        KQ_LAUNCH_CHECK("linear_targets_kernel");
    }
    Job j = {};
    j.T = T, j.V = V, j.d = d;
    j.target = target;
    j.lse = lse, j.entropy = entropy, j.g_logp = g_logp, j.g_entropy = g_entropy;
    j.ld_delta = c.piece;
    j.sum = reinterpret_cast<float*>(at + al256(c.delta) * (c.pieces > 1 ? 2 : 1));
    j.splits = c.splits, j.split_slabs = c.split_slabs;
    j.m_main = j.m_prod = static_cast<int32_t>(cdiv(T, BM));
    j.n_d = static_cast<int32_t>(cdiv(d, BN));
    j.d_slabs = static_cast<int32_t>(cdiv(d, BK));
    j.row_slabs = static_cast<int32_t>(cdiv(T, BK));
    j.info = info;
    bool fused = false;   // few rows: gW is done with D
    if (thin) {
        Maps t = m;
        KQ_TRY(make_map(&t.x, x, T, d, ldx, who, thin_box_rows(n)));
        // with few tiles of W its gradient goes by the tiles of gx's launch, which there are more of
        fused = gw && V >= kFused;
        j.delta = gx || !fused ? delta[0] : nullptr;
        j.gw = fused;
        KQ_TRY(run_thin_grad(t, j, stream));
        if (!gx && fused) return KQ_OK;
    }
    // launch i: D of piece i, the products with D of piece i - 1; of few rows gx alone is left
    for (int64_t i = 0; i <= c.pieces; ++i) {
        j.v_main = i * c.piece;
        j.w_main = std::min(c.piece, V - j.v_main);
        j.n_main = i < c.pieces && !thin ? static_cast<int32_t>(cdiv(j.w_main, BN)) : 0;
        j.delta = delta[i & 1];
        j.turned = thin;
        j.t_gx = j.t_gw = 0;
        if (i > 0) {
            j.v_prod = (i - 1) * c.piece;
            j.w_prod = std::min(c.piece, V - j.v_prod);
            j.prod_slabs = static_cast<int32_t>(cdiv(j.w_prod, BK));
            const int32_t splits = static_cast<int32_t>(cdiv(j.prod_slabs, c.split_slabs));
            j.first = i == 1;
            j.last = c.splits == 1 && i == c.pieces;
            if (gx) j.t_gx = splits * j.m_main * j.n_d;
            if (gw && !fused) j.t_gw = static_cast<int32_t>(cdiv(j.w_prod, BM)) * j.n_d;
        }
        j.tiles = j.t_gx + j.t_gw + j.m_main * j.n_main;
        m.d = read[(i + 1) & 1], m.out_d = write[i & 1];
        KQ_TRY(run_tiles<kDelta>(m, j, stream));
    }
    if (gx && c.splits > 1) {
        const int64_t blocks = std::min<int64_t>(cdiv(T * (d / 4), 64), static_cast<int64_t>(num_sms()) * 16);
        KQ_CUDA(launch_after(linear_gx_kernel, dim3(static_cast<unsigned>(blocks)), dim3(64), 0, stream,
                             static_cast<const float*>(j.sum), c.splits, T, d, reinterpret_cast<__nv_bfloat16*>(gx), ldgx));
        count_launch();
    }
    return KQ_OK;
}
