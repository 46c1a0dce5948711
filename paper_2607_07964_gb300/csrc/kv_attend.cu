// kq_kv_attend: attention of a few query rows over the 4-bit cache, one pass over the cached bytes.
//
// Mathematics. With a key k_j = s_j c_j + o_j (codes c in 0 .. 15) the score is
//     <q, k_j> = s_j <q, c_j> + o_j sum(q),
// so the tensor cores multiply q with the codes themselves and the grid enters as two numbers a
// row. The values likewise: sum_j p_j v_j = sum_j (p_j s'_j) c'_j + sum_j p_j o'_j. A nibble masked
// out of a word in place is the fp16 subnormal c 2^-24 (or 16 c 2^-24 four bits up), which
// mma.sync multiplies exactly, so a code costs about half an integer instruction and no conversion.
//   * q is scaled by a power of two into fp16: exact for bf16; fp32 is split into two fp16 halves
//     (22 bits), as are the weights p s' when the output is fp32. All sums are fp32.
//   * Codes enter about their middle, c - 8, so that the sums stay of the size of what they sum to: with
//     codes all positive the tensor cores' truncation adds up in one direction. For bf16 outputs the
//     scores' accumulators start at -8 sum(q) and the values' take -8 times the weights' sum (one more
//     product, with a constant) along with the rescaling that a new maximum needs. fp32 outputs
//     make c - 8 itself (two more instructions for four codes), and round each tile's sum into the
//     running one: 1e-6 of the output instead of 1e-4 over 2600 slots.
//   * p_j s'_j is scaled by a power of two of the row's own, which follows the largest such product (not the
//     largest s': a row of values that gets no weight says nothing about the ones that do) and keeps it
//     between 2^9 and 2^15: fp16 then holds the others to 11 bits over 23 binades below it, whatever the
//     values' range, and what is below counts for less than 2^-33 of the largest. (One unit for all rows, from the largest
//     s', is 1 % faster: 84.8 against 85.7 us for 64 sequences of up to 8192 slots.)
//
// What bounds it: the cache is read once, D + 8 bytes for each token and head; with D = 128 that
// leaves an SM 5.8 cycles a token at 6.8 TB/s, against ~3 issue slots and 1 to 2 tensor cycles, so
// the kernel is laid out to keep bulk copies in flight. A row of 16-byte units per token lets each
// lane take its operands straight from the staged bytes in the mma layout (a lane's 16 bytes of a
// key row are its share of every k step; the order of the dimensions inside a product is free).
//
// Split. The work is the list of 32-token steps of every item, a (sequence, head, group of query
// rows), each led by kItemCost steps that stand for its beginning and end (or the items of short
// sequences would all fall to a few warps). Each warp takes an equal, contiguous part of it, so ragged
// lengths, few sequences and long ones all fill the GPU evenly, without the host knowing the
// lengths. A warp streams its tokens through a ring of bulk copies that it refills itself and
// shares nothing with the other warps: 16 of them on an SM, none waiting for another. One that
// covers all of an item writes its output; parts are joined by kv_combine_kernel from at most two
// partial results a warp. (Four warps that shared tiles and joined their sums in shared memory lost
// about 10 us at every change of sequence.) Accumulated weights need the finished log-sum, so the
// scores are kept and kv_weight_kernel turns them into weights: 8 bytes a slot and row, written
// and read, in exchange for not reading the keys twice.
//
// With a window (kq_kv_attend_window) an item's steps are those of the first slots and those in which the windows of its rows can
// lie: as many for every group of rows of a sequence, so the list of work stays arithmetic; where the second lot begins is
// the group's own. Granules that no row sees are neither looked up nor copied.
//
// Measured, 64 query heads on 8, D = 128, bf16: 64 windows of 4096 in sequences of up to 32768 (285 MB) 73 us; 64 sequences of up to 8192 slots (360 MB) 78 us for
// the kernel, of which the copies run 58 us at 6.2 TB/s and the rest is its start and the spread of the
// warps' ends; 85 us with the joining. 16 of up to 131072 slots (1.44 GB) 271 us, 5.3 TB/s; 286 us where it keeps scores.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "kv_common.cuh"
#include "pdl.cuh"

namespace kq {
namespace {

constexpr int kWarps = 4;
constexpr int kStep = 2 * kGranule;             // tokens of a step
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 3;                       // steps in a warp's ring
constexpr int kAhead = 16;                       // steps whose addresses the lanes of a warp hold, a granule each
constexpr int kMaxRows = 40960;                  // rows of all pieces together: the workspace holds two results of each
constexpr int kMinSteps = 2;                     // of a piece, where there is little work
constexpr int kShortPart = 8;                    // steps, see the kernel
constexpr int kItemCost = 4;                     // what beginning and ending an item costs, in steps
constexpr float kSlack = 8.0f;                   // how far, in powers of two, a weight may pass 1
constexpr float kNone = -3.0e38f;                // a maximum over nothing: finite, so that differences with it are numbers
constexpr uint32_t kTopUnit = 127 + 126;         // the largest power of two that p s' enters with, biased
constexpr int kSettle = 8;                       // steps whose middle-code sums are taken off at once
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t y;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
// Of both halves; a NaN gives way to a number.
__device__ __forceinline__ uint32_t max_f16(uint32_t x, uint32_t y) {
    uint32_t z;
    asm("max.f16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y));
    return z;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
// Two codes of a word, nibbles 0 and 4 of x (ODD: 1 and 5), as the A operand. Plain: the masked
// bits, subnormals c 2^-24 (ODD: 16 c 2^-24). CENTRED: c - 8, through 1024 + c (ODD: 1024 + 16 c, over 16): the well-known
// way from small whole numbers to floats, their bits in the mantissa of a power of two that is then taken off.
template <bool CENTRED, bool ODD>
__device__ __forceinline__ uint32_t codes(uint32_t x) {
    constexpr uint32_t mask = ODD ? 0x00F000F0u : 0x000F000Fu;
    if constexpr (!CENTRED) return x & mask;
    uint32_t y = (x & mask) | 0x64006400u;
    if constexpr (ODD) asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(y) : "r"(0x2C002C00u), "r"(0xD480D480u));   // / 16 - 72
    else asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(y) : "r"(0x64086408u));                                      // - 1032
    return y;
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// 8 consecutive values; vec: they can be read 16 bytes at a time.
__device__ __forceinline__ void load8(const float* p, bool vec, float (&x)[8]) {
    if (vec) {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = p[i];
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, bool vec, float (&x)[8]) {
    if (vec) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(p[i]);
    }
}

struct Attend {
    KvView c;
    const void* q;
    int64_t tokens, q_token, q_head;   // strides in elements
    int32_t q_heads, group;            // query heads in all, and of a key/value head
    bool q_vec;                        // rows of q can be read 16 bytes at a time
    const int32_t* start;
    const int32_t* lens;
    float scale;
    void* out;
    float* lse;                        // [T][q_heads]
    float* scores;                     // [T][kv_heads][S][group], in units of ln 2, or nullptr
    int64_t S;
    int64_t cap;                       // slots a sequence may have: the table's, and S with weights
    struct Joint* joint;               // of each item in the list of work
    int64_t* items;                    // how many there are
    int64_t most_items;                // as many as the sequences of an ordered start can make
    int32_t window, sink;              // with a window: a token sees its last `window` slots and the first `sink`
    float* part;                       // [2 pieces][rows][D + 2]: sums, maximum, sum of weights
    int* info;
};

// What the warp that begins the rows of an item leaves to kv_combine_kernel.
struct Joint {
    int32_t first, last;     // the pieces that share them; equal: nothing to join
    int32_t h, row, rows;    // head, first query row of the sequence, number of rows
    int32_t token;           // the sequence's first token
};

// Steps that hold the slots that stay visible.
__device__ __forceinline__ int64_t first_steps(const Attend& p) { return (static_cast<int64_t>(p.sink) + kStep - 1) / kStep; }

// Sequence b's share of the work.
struct Seq {
    int32_t nq, rows_tiles, steps;   // queries, groups of ROWS query rows, steps (at least 1)
    int32_t n;                       // length
    int32_t first;                   // its first token
};
template <int ROWS, bool WINDOW>
__device__ __forceinline__ Seq sequence(const Attend& p, int b, int* info) {
    Seq s;
    const int64_t s0 = p.start[b], s1 = p.start[b + 1];
    s.n = static_cast<int32_t>(kv_length(p.lens, b, p.cap, info));
    s.first = static_cast<int32_t>(s0);
    s.nq = static_cast<int32_t>(s1 - s0);
    if (s0 < 0 || s1 < s0 || s1 > p.tokens) {
        record_error(info, -KQ_ERR_INVALID_ARG);
        s.nq = 0;
    }
    s.rows_tiles = static_cast<int32_t>((static_cast<int64_t>(s.nq) * p.group + ROWS - 1) / ROWS);
    s.steps = max(1, (s.n + kStep - 1) / kStep);
    if constexpr (WINDOW) {
        // ROWS rows are of at most this many tokens; their windows together, wherever they begin, and the first slots lie in
        // `most` steps
        const int64_t tokens = min(static_cast<int64_t>(s.nq), static_cast<int64_t>((ROWS - 2) / p.group + 2));
        const int64_t most = first_steps(p) + (p.window + tokens - 1 + 2 * (kStep - 1)) / kStep;
        s.steps = static_cast<int32_t>(min(static_cast<int64_t>(s.steps), most));
    }
    return s;
}
struct Work {
    int64_t steps, items;
};
__device__ __forceinline__ Work work_of(const Attend& p, const Seq& s) {
    const int64_t items = static_cast<int64_t>(s.rows_tiles) * p.c.kv_heads;
    return {items * (s.steps + kItemCost), items};
}
// Divisions of numbers that nearly always fit 32 bits.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}
// The slots that query token i (of nq) of a sequence with n slots sees.
__device__ __forceinline__ int32_t visible(int32_t n, int32_t nq, int32_t i) { return max(0, n - (nq - 1 - i)); }
// W steps in C pieces, the first r of them one longer: the first step of piece c, the piece of step w.
struct Pieces {
    int64_t q, r;
    __device__ Pieces(int64_t W, int64_t C) : q(divide(W, C)), r(W - q * C) {}
    __device__ int64_t first(int64_t c) const { return c * q + min(c, r); }
    __device__ int64_t of(int64_t w) const { return w < r * (q + 1) ? divide(w, q + 1) : r + divide(w - r * (q + 1), q); }
};

// lead: the sum of v over the threads before this one; returns the sum over all.
__device__ __forceinline__ Work scan_add(const Work& v, Work* tmp, Work& lead) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Work x = v, all = {0, 0};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x.steps, o), z = __shfl_up_sync(0xffffffffu, x.items, o);
        if (lane >= o) x.steps += y, x.items += z;
    }
    if (lane == 31) tmp[warp] = x;
    __syncthreads();
    lead = {x.steps - v.steps, x.items - v.items};
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) {
        if (i < warp) lead.steps += tmp[i].steps, lead.items += tmp[i].items;
        all.steps += tmp[i].steps, all.items += tmp[i].items;
    }
    return all;
}

// A position in the list of work: step `step` of row group `rt` of head h of sequence b.
struct Place {
    int b, h, rt;
    int v;          // place in the item's kItemCost + steps
    int step;       // the step that the warp's part of the item begins with
    int skip, turn; // with a window: steps from `turn` on lie `skip` steps further on in the sequence
    int low;        // and the first slot that a window of the item's rows holds
    int64_t item;   // its number in the list
    Seq s;
};
template <int ROWS, bool WINDOW>
__device__ __forceinline__ void next_sequence(const Attend& p, Place& at) {
    do {
        ++at.b;
        if (at.b >= p.c.batch) return;
        at.s = sequence<ROWS, WINDOW>(p, at.b, nullptr);
    } while (at.s.rows_tiles == 0);
}
// Past the rest of this row group.
template <int ROWS, bool WINDOW>
__device__ __forceinline__ void next_item(const Attend& p, Place& at) {
    at.v = 0;
    ++at.item;
    if (++at.rt < at.s.rows_tiles) return;
    at.rt = 0;
    if (++at.h < p.c.kv_heads) return;
    at.h = 0;
    next_sequence<ROWS, WINDOW>(p, at);
}

template <typename T, int D, int NT>
struct Shape {
    static constexpr int kRows = 8 * NT;
    static constexpr int kGranuleBytes = kGranule * (D + 8);
    static constexpr int kStageBytes = 2 * kGranuleBytes;
    static constexpr size_t kSmem = kWarps * kStages * kStageBytes;
    // CTAs on an SM: what the sums, twice as many with 16 rows or 128 dimensions, leave of the registers
    static constexpr int kCtas = D == 64 ? (NT == 1 ? 5 : sizeof(T) == 4 ? 3 : 4) : (NT == 1 ? 4 : sizeof(T) == 4 ? 2 : 3);
};

// A warp's state for a group of NT x 8 query rows. A lane (g8, t4) has columns 2 t4 and
// 2 t4 + 1 of each 8 rows.
template <typename T, int D, int NT, bool WINDOW>
struct Rows {
    static constexpr bool kSplit = sizeof(T) == 4;   // fp32: two fp16 halves of q and of the weights
    static constexpr int kWords = D / 32;            // code words of a row that a lane of a quad takes
    uint32_t bq[NT][kWords][4], bl[NT][kSplit ? kWords : 1][4];   // q, and what fp16 left of it
    float alpha[NT][2], gamma[NT][2];                // score = alpha (s S + o gamma), S from the tensor cores
    int32_t lim[NT][2];                              // slots seen
    int32_t low[NT][2], sink;                        // with a window: of them from low on, and the first `sink`
    int64_t put[NT][2];                              // where scores go
    float o[NT][D / 16][4], m[NT][2], l[NT][2], off[NT][2];
    float mid[NT][4];                                // 8 times the sum of the weights in o (codes not centred)
    uint32_t unit[NT][2];                            // biased exponent of the power of two that p s' enters o with

    __device__ __forceinline__ bool sees(int nt, int k, int slot) const {
        return slot < lim[nt][k] && (!WINDOW || slot >= low[nt][k] || slot < sink);
    }
    // o = corr (o - mid), mid = 0
    __device__ __forceinline__ void settle_mid(int nt, const float (&corr)[2]) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (kSplit) o[nt][i][j] *= corr[j & 1];
                else o[nt][i][j] = corr[j & 1] * fmaf(j < 2 ? -1.0f : -16.0f, mid[nt][j], o[nt][i][j]);
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) mid[nt][j] = 0.0f;
    }

    // Two granules: 32 tokens from slot `slot`, staged at gr. MASK: some slot may be unseen by some row.
    // settle: take the middle code off the sums in any case.
    template <bool MASK>
    __device__ __forceinline__ void step(const uint8_t* gr, int slot, int g8, int t4, float* scores, int group, bool settle) {
        // the token of A row g8 (and 8 more of row g8 + 8), chosen so that the tokens 2 t4, 2 t4 + 1, 2 t4 + 8 and
        // 2 t4 + 9 of the weights' fragment are rows t4, 7 - t4, 8 + t4, 15 - t4: neighbouring lanes
        // then read neighbouring rows of codes
        const int tok = (g8 & 1) ? 7 - (g8 >> 1) : (g8 >> 1);
        constexpr int kBytes = kGranule * (D + 8);
        float s[2][NT][4], vs[2][2], vo[2][2];
#pragma unroll
        for (int gi = 0; gi < 2; ++gi) {
            const uint8_t* g = gr + gi * kBytes;
            // fp32: the two halves of the dimensions and the low part of q apart, as the tensor cores
            // truncate each sum to its own size
            float s2[NT][kSplit ? 2 : 1][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[gi][nt][j] = kSplit ? 0.0f : -8.0f * gamma[nt][j & 1];
                    s2[nt][0][j] = 0.0f;
                    if constexpr (kSplit) s2[nt][1][j] = 0.0f;
                }
            uint32_t ka[kWords], kb[kWords];
            if constexpr (D == 128) {
                const uint4 u = *reinterpret_cast<const uint4*>(g + tok * 64 + t4 * 16);
                const uint4 v = *reinterpret_cast<const uint4*>(g + (tok + 8) * 64 + t4 * 16);
                ka[0] = u.x, ka[1] = u.y, ka[2] = u.z, ka[3] = u.w;
                kb[0] = v.x, kb[1] = v.y, kb[2] = v.z, kb[3] = v.w;
            } else {
                const uint2 u = *reinterpret_cast<const uint2*>(g + tok * 32 + t4 * 8);
                const uint2 v = *reinterpret_cast<const uint2*>(g + (tok + 8) * 32 + t4 * 8);
                ka[0] = u.x, ka[1] = u.y;
                kb[0] = v.x, kb[1] = v.y;
            }
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const uint32_t x = hf ? ka[i] >> 8 : ka[i], y = hf ? kb[i] >> 8 : kb[i];
                    const uint32_t a0 = codes<kSplit, false>(x), a1 = codes<kSplit, false>(y);
                    const uint32_t a2 = codes<kSplit, true>(x), a3 = codes<kSplit, true>(y);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (kSplit) {
                            mma_f16(2 * i < kWords ? s[gi][nt] : s2[nt][0], a0, a1, a2, a3, bq[nt][i][2 * hf], bq[nt][i][2 * hf + 1]);
                            mma_f16(s2[nt][1], a0, a1, a2, a3, bl[nt][i][2 * hf], bl[nt][i][2 * hf + 1]);
                        } else {
                            mma_f16(s[gi][nt], a0, a1, a2, a3, bq[nt][i][2 * hf], bq[nt][i][2 * hf + 1]);
                        }
                    }
                }
            }
            const uint32_t* prm = reinterpret_cast<const uint32_t*>(g + kGranule * D);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                // the grid about its middle code: x = s (c - 8) + (o + 8 s)
                const uint32_t kp = prm[tok + 8 * hf], vp = prm[16 + tok + 8 * hf];
                const float ks = kv_scale(kp), ko = fmaf(8.0f, ks, kv_offset(kp));
                vs[gi][hf] = kv_scale(vp);
                vo[gi][hf] = fmaf(8.0f, vs[gi][hf], kv_offset(vp));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float& x = s[gi][nt][2 * hf + k];
                        if constexpr (kSplit) x += s2[nt][0][2 * hf + k] + s2[nt][1][2 * hf + k];
                        x = fmaf(ks, x, ko * gamma[nt][k]);
                        if (MASK && !sees(nt, k, slot + 16 * gi + tok + 8 * hf)) x = -INFINITY;
                    }
            }
        }
        if (scores) {
#pragma unroll
            for (int gi = 0; gi < 2; ++gi)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const int64_t sl = slot + 16 * gi + tok + 8 * hf;
                        const float x0 = alpha[nt][0] * s[gi][nt][2 * hf], x1 = alpha[nt][1] * s[gi][nt][2 * hf + 1];
                        if (!(group & 1)) {   // two columns are neighbours of one token
                            if (sl < lim[nt][0]) *reinterpret_cast<float2*>(scores + put[nt][0] + sl * group) = make_float2(x0, x1);
                        } else {
                            if (sl < lim[nt][0]) scores[put[nt][0] + sl * group] = x0;
                            if (sl < lim[nt][1]) scores[put[nt][1] + sl * group] = x1;
                        }
                    }
        }
        // The maximum that the weights are taken against, a whole number, moves only when a score passes it by 2^kSlack:
        // that is rare after the first tiles. The unit of p s' moves against it, so that the sums in o stay what they are
        // (but for the first maximum, and products below 2^-111, whose unit is the largest there is).
        float mx[NT][2];
        bool move = settle;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                mx[nt][k] = fmaxf(fmaxf(s[0][nt][k], s[0][nt][2 + k]), fmaxf(s[1][nt][k], s[1][nt][2 + k])) * alpha[nt][k];
                move |= mx[nt][k] > m[nt][k] + kSlack;
            }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float corr[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float x = mx[nt][k];
#pragma unroll
                    for (int sh = 4; sh < 32; sh <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, sh));
                    const float mn = fmaxf(m[nt][k], ceilf(x)), r = ex2(m[nt][k] - mn);
                    const uint32_t up = min(kTopUnit - unit[nt][k], static_cast<uint32_t>(fminf(mn - m[nt][k], 256.0f)));
                    corr[k] = ex2(m[nt][k] - mn + static_cast<float>(up));
                    unit[nt][k] += up;
                    m[nt][k] = mn;
                    l[nt][k] *= r;
                    off[nt][k] *= r;
                }
                settle_mid(nt, corr);
            }
        }
        // s = p s'
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int gi = 0; gi < 2; ++gi)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        float& x = s[gi][nt][2 * hf + k];
                        const float pr = ex2(fmaf(alpha[nt][k], x, -m[nt][k]));
                        l[nt][k] += pr;
                        if (MASK) {
                            const bool in = sees(nt, k, slot + 16 * gi + tok + 8 * hf);
                            off[nt][k] += in ? pr * vo[gi][hf] : 0.0f;
                            x = in ? pr * vs[gi][hf] : 0.0f;
                        } else {
                            off[nt][k] = fmaf(pr, vo[gi][hf], off[nt][k]);
                            x = pr * vs[gi][hf];
                        }
                    }
        // in fp16; where one passes 2^15, which is rare too, the rows' units come down and they are made again
        uint32_t b[2][NT][2], e[2][NT][2];
        for (bool again = true;; again = false) {
            uint32_t top = 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int gi = 0; gi < 2; ++gi)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const float u0 = __uint_as_float(unit[nt][0] << 23), u1 = __uint_as_float(unit[nt][1] << 23);
                        const uint32_t h = pack_f16(s[gi][nt][2 * hf] * u0, s[gi][nt][2 * hf + 1] * u1);
                        b[gi][nt][hf] = h;
                        top = max_f16(top, h);
                    }
            if (!again || !__any_sync(0xffffffffu, (top + 0x08000800u) & 0x80008000u)) break;   // either half from 2^15 up
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float corr[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float x = fmaxf(fmaxf(s[0][nt][k], s[0][nt][2 + k]), fmaxf(s[1][nt][k], s[1][nt][2 + k]));
#pragma unroll
                    for (int sh = 4; sh < 32; sh <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, sh));
                    const uint32_t low = min(unit[nt][k], 127 + 9 + 127 - (__float_as_uint(x) >> 23));   // x from 2^9 to 2^10
                    corr[k] = __uint_as_float(static_cast<uint32_t>(max(0, 127 - static_cast<int>(unit[nt][k] - low))) << 23);
                    unit[nt][k] = low;
                }
                settle_mid(nt, corr);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // weights of 16 tokens by 8 rows into the B fragment: token pairs along a lane
#pragma unroll
            for (int gi = 0; gi < 2; ++gi)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    if constexpr (kSplit) {
                        const float u0 = __uint_as_float(unit[nt][0] << 23), u1 = __uint_as_float(unit[nt][1] << 23);
                        const float2 f = unpack_f16(b[gi][nt][hf]);
                        e[gi][nt][hf] = transpose8(pack_f16(fmaf(s[gi][nt][2 * hf], u0, -f.x), fmaf(s[gi][nt][2 * hf + 1], u1, -f.y)));
                    }
                    b[gi][nt][hf] = transpose8(b[gi][nt][hf]);
                }
            if constexpr (!kSplit) {   // in every row of the accumulator's layout
#pragma unroll
                for (int gi = 0; gi < 2; ++gi)
                    mma_f16(mid[nt], 0x00080008u, 0x00080008u, 0x00080008u, 0x00080008u, b[gi][nt][0], b[gi][nt][1]);
            }
        }
        // values: words of dimensions 16 g8 .. (D = 128) or 8 g8 .. (D = 64) of four tokens
#pragma unroll
        for (int gi = 0; gi < 2; ++gi) {
            const uint8_t* vr = gr + gi * kBytes + kGranule * (D / 2) + g8 * (D / 16);
            uint32_t v[4][D / 64];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int tk = (i >> 1) * 8 + (i & 1 ? 7 - t4 : t4);
                if constexpr (D == 128) {
                    const uint2 u = *reinterpret_cast<const uint2*>(vr + tk * 64);
                    v[i][0] = u.x, v[i][1] = u.y;
                } else {
                    v[i][0] = *reinterpret_cast<const uint32_t*>(vr + tk * 32);
                }
            }
#pragma unroll
            for (int j = 0; j < D / 64; ++j)
#pragma unroll
                for (int qd = 0; qd < 4; ++qd) {   // dimensions 2 qd and 2 qd + 1 of the word
                    const uint32_t sel = qd < 2 ? 0x5410u : 0x7632u;
                    uint32_t x = __byte_perm(v[0][j], v[1][j], sel), y = __byte_perm(v[2][j], v[3][j], sel);
                    if (qd & 1) x >>= 8, y >>= 8;
                    const uint32_t a0 = codes<kSplit, false>(x), a1 = codes<kSplit, true>(x);
                    const uint32_t a2 = codes<kSplit, false>(y), a3 = codes<kSplit, true>(y);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float(&ac)[4] = o[nt][4 * j + qd];
                        if constexpr (kSplit) {   // 16 tokens' sum by itself, then rounded into the running one
                            float u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                            mma_f16(u, a0, a1, a2, a3, e[gi][nt][0], e[gi][nt][1]);
                            mma_f16(u, a0, a1, a2, a3, b[gi][nt][0], b[gi][nt][1]);
#pragma unroll
                            for (int r = 0; r < 4; ++r) ac[r] += u[r];
                        } else {
                            mma_f16(ac, a0, a1, a2, a3, b[gi][nt][0], b[gi][nt][1]);
                        }
                    }
                }
        }
    }
};

// The place in the sequence of an item's step.
template <bool WINDOW>
__device__ __forceinline__ int step_at(const Place& at, int step) {
    return WINDOW && step >= at.turn ? step + at.skip : step;
}

// A warp's ring of staged granules. Lane l holds the address of granule l & 1 of step l / 2 of the
// kAhead steps around the next load; the page numbers of the kAhead steps after them are on their
// way. A warp refills a stage when its lanes have read it, so no other warp is waited for.
template <int D, bool WINDOW>
struct Feed {
    static constexpr int kBytes = kGranule * (D + 8);
    const uint8_t* src;   // of this lane's granule
    int32_t next;         // its page number kAhead steps later

    __device__ __forceinline__ int slot_of(const Place& at, int k, int lane) const {
        return step_at<WINDOW>(at, at.step + k + (lane >> 1)) * kStep + (lane & 1) * kGranule;
    }
    // Whether a row may see a slot of the granule: others are not asked for, as their pages may be gone.
    __device__ __forceinline__ bool seen(const Attend& p, const Place& at, int slot) const {
        return slot < at.s.n && (!WINDOW || slot < p.sink || slot > at.low - kGranule);
    }
    // the page number of this lane's granule in the steps from k, of a segment of seg steps
    __device__ __forceinline__ int32_t fetch(const Attend& p, const Place& at, int k, int seg, int lane) const {
        const int slot = slot_of(at, k, lane);
        if (k + (lane >> 1) >= seg || !seen(p, at, slot)) return 0;
        const int32_t id = p.c.table[static_cast<int64_t>(at.b) * p.c.table_ld + slot / p.c.page];
        if (id >= 0 && id < p.c.pages) return id;
        record_error(p.info, -KQ_ERR_INVALID_ARG);
        return 0;
    }
    __device__ __forceinline__ void place(const Attend& p, const Place& at, int k, int32_t id, int lane) {
        const int slot = slot_of(at, k, lane);
        src = p.c.data + (static_cast<int64_t>(id) * p.c.kv_heads + at.h) * kv_head_bytes(p.c) + slot % p.c.page * (D + 8);
    }
    // Step k's granules into a stage (k < seg). Both are one run unless a page can end between them.
    __device__ __forceinline__ void load(const Attend& p, const Place& at, int k, int seg, uint8_t* stage, uint64_t* bar, int lane) {
        if (k % kAhead == 0 && k > 0) {
            place(p, at, k, next, lane);
            next = fetch(p, at, k + kAhead, seg, lane);
        }
        const int slot = step_at<WINDOW>(at, at.step + k) * kStep;
        const bool one = seen(p, at, slot), two = seen(p, at, slot + kGranule);
        const int many = one + two;
        const uint64_t a = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(src), 2 * (k % kAhead));
        uint64_t a2 = a + kBytes;
        if (WINDOW || p.c.page % (2 * kGranule)) a2 = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(src), 2 * (k % kAhead) + 1);
        if (lane == 0) {
            if (many == 0) {
                mbar_arrive(bar);
            } else {
                mbar_arrive_expect_tx(bar, many * kBytes);
                const bool run = many == 1 || a2 == a + kBytes;
                if (!WINDOW || one) bulk_load(stage, reinterpret_cast<const void*>(a), run ? many * kBytes : kBytes, bar);
                if (!run || (WINDOW && !one)) bulk_load(stage + kBytes, reinterpret_cast<const void*>(a2), kBytes, bar);
            }
        }
        __syncwarp();
    }
};

template <typename T, int D, int NT, bool WINDOW>
__global__ void __launch_bounds__(kThreads, Shape<T, D, NT>::kCtas) kv_attend_kernel(const Attend p) {
    using Sh = Shape<T, D, NT>;
    constexpr int kRows = Sh::kRows;
    constexpr bool kSplit = Rows<T, D, NT, WINDOW>::kSplit;
    constexpr int kWords = Rows<T, D, NT, WINDOW>::kWords;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t full[kWarps][kStages];
    __shared__ int abort_flag[kWarps];
    __shared__ Work scan_tmp[kWarps], found_base[kWarps];
    __shared__ int found_b[kWarps];
    __shared__ Seq found_s[kWarps];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const KvView& c = p.c;

    // ---- this warp's part of the work
    if (lane == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(&full[warp][i], 1);
        fence_mbar_init();
        abort_flag[warp] = 0;
        found_b[warp] = -1;
    }
    pdl_wait();   // nothing before this reads or writes global memory
    if (blockIdx.x == 0 && tid == 0 && (p.start[0] != 0 || p.start[c.batch] != p.tokens)) record_error(p.info, -KQ_ERR_INVALID_ARG);
    // the sequences' steps, a run of sequences to a thread: the total, then the sequence that holds a warp's first
    const int run = (c.batch + kThreads - 1) / kThreads, b0 = min(tid * run, c.batch), b1 = min(b0 + run, c.batch);
    Work v = {0, 0}, lead;
    for (int b = b0; b < b1; ++b) {
        const Work one = work_of(p, sequence<kRows, WINDOW>(p, b, blockIdx.x ? nullptr : p.info));
        v.steps += one.steps, v.items += one.items;
    }
    const Work all = scan_add(v, scan_tmp, lead);
    const int64_t W = all.steps;
    const int64_t C = max(static_cast<int64_t>(1), min(static_cast<int64_t>(gridDim.x) * kWarps, (W + kMinSteps - 1) / kMinSteps));
    const Pieces pieces(W, C);
    const int64_t me = warp * static_cast<int64_t>(gridDim.x) + blockIdx.x;   // neighbours in the list on different SMs
    const int64_t w0 = me < C ? pieces.first(me) : W, w1 = me < C ? pieces.first(me + 1) : W;
    if (blockIdx.x == 0 && tid == 0) *p.items = all.items;
    for (int i = 0; i < kWarps; ++i) {
        const int64_t other = i * static_cast<int64_t>(gridDim.x) + blockIdx.x;
        const int64_t o0 = other < C ? pieces.first(other) : W;
        if (o0 < lead.steps || o0 >= lead.steps + v.steps) continue;
        Work at = lead;
        for (int b = b0; b < b1; ++b) {
            const Seq s = sequence<kRows, WINDOW>(p, b, nullptr);
            const Work one = work_of(p, s);
            if (o0 < at.steps + one.steps) {
                found_b[i] = b;
                found_base[i] = at;
                found_s[i] = s;
                break;
            }
            at.steps += one.steps, at.items += one.items;
        }
    }
    __syncthreads();
    pdl_launch_dependents();
    if (w0 >= w1 || found_b[warp] < 0) return;   // from here on the warps are on their own
    Place at;
    at.b = found_b[warp];
    at.s = found_s[warp];
    {
        const int64_t rem = w0 - found_base[warp].steps, length = at.s.steps + kItemCost, head = at.s.rows_tiles * length;
        at.h = static_cast<int>(divide(rem, head));
        at.rt = static_cast<int>(divide(rem - at.h * head, length));
        at.v = static_cast<int>(rem - at.h * head - at.rt * length);
        at.item = found_base[warp].items + static_cast<int64_t>(at.h) * at.s.rows_tiles + at.rt;
    }

    const int g8 = lane >> 2, t4 = lane & 3;
    uint8_t* const ring = smem + warp * kStages * Sh::kStageBytes;
    int it = 0;        // steps of this warp so far: its stage and the parity of its barrier
    bool fine_waits = true;   // a wait that gave up ends the warp's work
    int issued = 0;
    for (int64_t w = w0; w < w1 && fine_waits;) {
        // this warp's part of the item: steps from at.step, seg of them
        const int length = at.s.steps + kItemCost, part_of = static_cast<int>(min(w1 - w, static_cast<int64_t>(length - at.v)));
        at.step = max(at.v - kItemCost, 0);
        const int seg = max(at.v + part_of - kItemCost, 0) - at.step;
        if (seg == 0) break;   // the warp's last, and the next warp's item
        const int rows = min(kRows, at.s.nq * p.group - at.rt * kRows);
        const int least = visible(at.s.n, at.s.nq, at.rt * kRows / p.group);   // what the first row's token has before it
        if constexpr (WINDOW) {
            at.low = max(0, least - p.window);
            at.turn = static_cast<int>(min(first_steps(p), static_cast<int64_t>(at.s.steps)));
            at.skip = max(0, min(at.low / kStep - at.turn, (at.s.n + kStep - 1) / kStep - at.s.steps));
        }
        if (at.step == 0 && lane == 0) {
            Joint j;
            j.first = static_cast<int32_t>(me);
            j.last = seg == at.s.steps ? j.first : static_cast<int32_t>(pieces.of(w - at.v + length - 1));
            j.h = at.h;
            j.row = at.rt * kRows;
            j.rows = rows;
            j.token = at.s.first;
            if (at.item < p.most_items && KQ_IN_RANGE(at.item, p.most_items)) p.joint[at.item] = j;
            else record_error(p.info, -KQ_ERR_INVALID_ARG);   // sequences that overlap
        }
        Feed<D, WINDOW> feed;
        const int32_t page_id = feed.fetch(p, at, 0, seg, lane);
        feed.next = feed.fetch(p, at, kAhead, seg, lane);
        Rows<T, D, NT, WINDOW> R;
        float xs[NT][kWords][8];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = at.rt * kRows + min(nt * 8 + g8, rows - 1);   // rows past the last repeat it; their results are not used
            const T* src = static_cast<const T*>(p.q) + (at.s.first + r / p.group) * p.q_token +
                           (static_cast<int64_t>(at.h) * p.group + r % p.group) * p.q_head + t4 * (D / 4);
#pragma unroll
            for (int i = 0; i < kWords; ++i) load8(src + 8 * i, p.q_vec, xs[nt][i]);
        }
        feed.place(p, at, 0, page_id, lane);
#pragma unroll
        for (int k = 0; k < kStages; ++k)
            if (k < seg) {
                const int stage = issued++ % kStages;
                feed.load(p, at, k, seg, ring + stage * Sh::kStageBytes, &full[warp][stage], lane);
            }
        // q: lane (g8, t4) holds dimensions t4 D / 4 .. of row g8, each word of 8 as two k steps: (0, 4 | 1, 5) and
        // (2, 6 | 3, 7); the odd ones are divided by 16 where their nibbles sit four bits up
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float sum = 0.0f;
            uint32_t top = 0;   // as bits: an infinity or a NaN is above every number
#pragma unroll
            for (int i = 0; i < kWords; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    top = max(top, __float_as_uint(xs[nt][i][j]) & 0x7FFFFFFFu);
                    sum += xs[nt][i][j];
                }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            const bool bad = top >= 0x7F800000u;
            // 2^e brings the largest below 2^14; both powers stay normal. The sign of the scale goes to q, so that
            // alpha > 0 and scores compare before they are scaled.
            const int e = min(100, max(-113, 13 - static_cast<int>(top >> 23) + 127));
            const float up = copysignf(__uint_as_float(static_cast<uint32_t>(e + 127) << 23), p.scale);
            const float f = fmaxf(fabsf(p.scale) * kLog2e, 0x1p-126f);
            // score / ln 2 = f (s sum(q c) + o sum(q)) with sum(q c) = S / unit
            const float unit = kSplit ? up : up * 0x1p-24f;
            const float a = bad ? NAN : fmaxf((kSplit ? f : f * 0x1p24f) * __uint_as_float(static_cast<uint32_t>(127 - e) << 23), 0x1p-126f);
            const float gm = bad ? 0.0f : sum * unit;
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const float(&x)[8] = xs[nt][i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {   // nibbles j and j + 4
                    const float s = up * (!kSplit && (j & 1) ? 0.0625f : 1.0f);
                    const float x0 = bad ? 0.0f : x[j] * s, x1 = bad ? 0.0f : x[j + 4] * s;
                    R.bq[nt][i][j] = pack_f16(x0, x1);
                    if constexpr (kSplit) {
                        const float2 h = unpack_f16(R.bq[nt][i][j]);
                        R.bl[nt][i][j] = pack_f16(x0 - h.x, x1 - h.y);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {   // the accumulator's columns 2 t4 + k
                const int col = nt * 8 + 2 * t4 + k, crow = at.rt * kRows + col;
                R.alpha[nt][k] = __shfl_sync(0xffffffffu, a, (2 * t4 + k) * 4);
                R.gamma[nt][k] = __shfl_sync(0xffffffffu, gm, (2 * t4 + k) * 4);
                const int i = crow / p.group;
                R.lim[nt][k] = col < rows ? visible(at.s.n, at.s.nq, i) : 0;
                if constexpr (WINDOW) R.low[nt][k] = R.lim[nt][k] - p.window, R.sink = p.sink;
                R.put[nt][k] = ((static_cast<int64_t>(at.s.first + i) * c.kv_heads + at.h) * p.S) * p.group + crow % p.group;
                R.m[nt][k] = kNone, R.l[nt][k] = 0.0f, R.off[nt][k] = 0.0f, R.unit[nt][k] = kTopUnit;
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) R.o[nt][i][j] = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) R.mid[nt][j] = 0.0f;
        }
        // The steps that every row sees in full, then those with an end: two loops, so that the first one
        // carries its sums in place.
        auto turn = [&](int k, auto masked) {
            const int stage = it % kStages;
            uint8_t* gr = ring + stage * Sh::kStageBytes;
            uint64_t* bar = &full[warp][stage];
            if (__any_sync(0xffffffffu, !mbar_try_wait(bar, (it / kStages) & 1)))
                fine_waits = __all_sync(0xffffffffu, mbar_wait(bar, (it / kStages) & 1, &abort_flag[warp]));
            const int slot = step_at<WINDOW>(at, at.step + k) * kStep;
            if (fine_waits && (!decltype(masked)::value || slot < at.s.n))   // uniform over the warp
                R.template step<decltype(masked)::value>(gr, slot, g8, t4, p.scores, p.group, k % kSettle == 0);
            __syncwarp();
            if (fine_waits && k + kStages < seg) {
                feed.load(p, at, k + kStages, seg, gr, bar, lane);
                ++issued;
            }
            ++it;
        };
        // With a window parts are short and the code of a step is large: what waits is the fetch of instructions. So one loop for the
        // steps at both ends, and for all of a short part (24 drafts in windows of 515, fp32: 27.9 us with three loops, 23.3 with two,
        // 21.1 with one for parts below 8 steps, as below 6 or 12; 64 windows of 4096 72.8, 73.9 and 74.0).
        const int whole_steps = WINDOW && seg < kShortPart ? 0 : min(seg, least / kStep - at.step - (WINDOW ? at.skip : 0));
        int k = 0;
        if constexpr (WINDOW) {
            // steps with first slots or a window's beginning, the last row's the latest, then whole ones, then those with an end
            const int begin = visible(at.s.n, at.s.nq, (at.rt * kRows + rows - 1) / p.group) - p.window;
            const int clear = begin <= 0 ? 0 : max(at.turn, (begin + kStep - 1) / kStep - at.skip) - at.step;
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {
                for (const int end = pass ? seg : min(seg, clear); k < end && fine_waits; ++k) turn(k, std::true_type());
                for (; k < whole_steps && fine_waits; ++k) turn(k, std::false_type());
            }
        } else {
            for (; k < whole_steps && fine_waits; ++k) turn(k, std::false_type());
            for (; k < seg && fine_waits; ++k) turn(k, std::true_type());
        }
        if (!fine_waits) break;

        // ---- the rows' result, or this piece's part of it
        const bool whole = seg == at.s.steps;
        float* part = p.part + (2 * me + (at.step == 0)) * (kRows * (D + 2));   // of an item begun here, of one gone on with
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float one[2] = {1.0f, 1.0f};
            if constexpr (!kSplit) R.settle_mid(nt, one);
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                float L = R.l[nt][k2], off = R.off[nt][k2];
#pragma unroll
                for (int sh = 4; sh < 32; sh <<= 1) {
                    L += __shfl_xor_sync(0xffffffffu, L, sh);
                    off += __shfl_xor_sync(0xffffffffu, off, sh);
                }
                const int col = nt * 8 + 2 * t4 + k2;
                if (col >= rows) continue;
                // the unit taken back, with 2^24 of subnormal codes; what float32 cannot hold of it, for products of
                // 2^113 and more, goes to the sums first
                const int power = 127 - static_cast<int>(R.unit[nt][k2]) + (kSplit ? 0 : 24), past = max(0, power - 127);
                const float up = __uint_as_float(static_cast<uint32_t>(power - past + 127) << 23);
                const float first = __uint_as_float(static_cast<uint32_t>(past + 127) << 23);
                if (!KQ_IN_RANGE(part + kRows * (D + 2) - 1 - p.part, 2ll * kMaxRows * (D + 2))) continue;
                float x[D / 8];   // dimensions g8 D / 8 ..
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    x[2 * i] = fmaf(R.o[nt][i][k2] * first, up, off);
                    x[2 * i + 1] = fmaf(R.o[nt][i][2 + k2] * first, kSplit ? up : up * 0.0625f, off);
                }
                if (whole) {
                    const int row = at.rt * kRows + col;
                    const int64_t r = (static_cast<int64_t>(at.s.first) + row / p.group) * p.q_heads + at.h * p.group + row % p.group;
                    if (!KQ_IN_RANGE(r, p.tokens * p.q_heads)) continue;
                    T* dst = static_cast<T*>(p.out) + r * D + g8 * (D / 8);
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) dst[i] = static_cast<T>(L == 0.0f ? 0.0f : x[i] * inv);
                    if (g8 == 0 && p.lse) p.lse[r] = L == 0.0f ? -INFINITY : (R.m[nt][k2] + log2f(L)) * kLn2;
                } else {
                    float4* dst = reinterpret_cast<float4*>(part + col * D + g8 * (D / 8));
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) dst[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    if (g8 == 0) {
                        part[kRows * D + col] = R.m[nt][k2];
                        part[kRows * (D + 1) + col] = L;
                    }
                }
            }
        }
        w += part_of;
        at.v += part_of;
        if (at.v == length) next_item<kRows, WINDOW>(p, at);
    }
    if (!fine_waits && lane == 0) {   // leave only when this warp's copies have landed
        record_error(p.info, -KQ_ERR_TIMEOUT);
        int none = 0;
        for (int i = max(0, issued - kStages); i < issued; ++i) mbar_wait(&full[warp][i % kStages], (i / kStages) & 1, &none);
    }
}

// Joins the partial results of rows that more than one warp worked on: blocks (i, ..) for item i. A warp
// takes a column, its lanes four dimensions each (D = 64: two); where the results are many, a block
// takes a column and its warps share them.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(256) kv_combine_kernel(const Attend p) {
    constexpr int kRows = 8 * NT, kV = D / 32, kGroups = 8;
    constexpr int64_t kPart = kRows * (D + 2);
    __shared__ float sm[kGroups][D], sl[kGroups], sx[kGroups];
    pdl_wait();
    pdl_launch_dependents();
    const int64_t items = *p.items;
    const Joint j = p.joint[blockIdx.x];   // the array has room for every block
    if (blockIdx.x >= items || j.last == j.first) return;
    // a warp that gave up leaves items undescribed
    if (j.first < 0 || j.last < j.first || j.last >= kMaxRows / kRows || j.h < 0 || j.h >= p.c.kv_heads || j.row < 0 || j.rows < 1 ||
        j.rows > kRows || j.token < 0 || j.token + (static_cast<int64_t>(j.row) + j.rows - 1) / p.group >= p.tokens)
        return;
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const int many = j.last - j.first + 1;
    // the piece that begins the item has its result second, those that go on with it first
    auto result = [&](int k) { return p.part + (2 * static_cast<int64_t>(j.first + k) + (k == 0)) * kPart; };
    const bool share = many > 32;
    for (int col = share ? blockIdx.y : grp + blockIdx.y * kGroups; col < j.rows; col += gridDim.y * (share ? 1 : kGroups)) {
        float M = kNone, L = 0.0f, O[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) O[i] = 0.0f;
        for (int k = (share ? grp * 32 : 0) + lane; k < many; k += share ? 256 : 32) M = fmaxf(M, result(k)[kRows * D + col]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        if (share) {
            __syncthreads();
            if (lane == 0) sx[grp] = M;
            __syncthreads();
#pragma unroll
            for (int g = 0; g < kGroups; ++g) M = fmaxf(M, sx[g]);
        }
        for (int k0 = share ? grp * 32 : 0; k0 < many; k0 += share ? 256 : 32) {
            const int here = min(32, many - k0);
            float f = 0.0f;
            if (lane < here) {
                const float* q = result(k0 + lane);
                f = ex2(q[kRows * D + col] - M);
                L = fmaf(f, q[kRows * (D + 1) + col], L);
            }
            constexpr int kAhead = 16;   // results in flight
            for (int k1 = 0; k1 < here; k1 += kAhead) {
                float x[kAhead][kV];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (k1 + k >= here) break;
                    const float* q = result(k0 + k1 + k) + col * D + lane * kV;
                    if constexpr (kV == 4) {
                        const float4 y = *reinterpret_cast<const float4*>(q);
                        x[k][0] = y.x, x[k][1] = y.y, x[k][2] = y.z, x[k][3] = y.w;
                    } else {
                        const float2 y = *reinterpret_cast<const float2*>(q);
                        x[k][0] = y.x, x[k][1] = y.y;
                    }
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    if (k1 + k >= here) break;
                    const float fk = __shfl_sync(0xffffffffu, f, k1 + k);
#pragma unroll
                    for (int i = 0; i < kV; ++i) O[i] = fmaf(fk, x[k][i], O[i]);
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
        if (share) {
#pragma unroll
            for (int i = 0; i < kV; ++i) sm[grp][lane * kV + i] = O[i];
            if (lane == 0) sl[grp] = L;
            __syncthreads();
            if (grp == 0)
                for (int g = 1; g < kGroups; ++g) {
                    L += sl[g];
#pragma unroll
                    for (int i = 0; i < kV; ++i) O[i] += sm[g][lane * kV + i];
                }
            __syncthreads();
            if (grp > 0) continue;
        }
        const int row = j.row + col;
        const int64_t r = (static_cast<int64_t>(j.token) + row / p.group) * p.q_heads + j.h * p.group + row % p.group;
        if (!KQ_IN_RANGE(r, p.tokens * p.q_heads)) continue;
        T* dst = static_cast<T*>(p.out) + r * D + lane * kV;
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
#pragma unroll
        for (int i = 0; i < kV; ++i) dst[i] = static_cast<T>(L == 0.0f ? 0.0f : O[i] * inv);
        if (lane == 0 && p.lse) p.lse[r] = L == 0.0f ? -INFINITY : (M + log2f(L)) * kLn2;
    }
}

// acc += the weights of the slots: a thread takes kSlots of them, the rows of their sequence and head in
// order. Bound by the scores' bytes, 4 a row, so what counts is loads in flight: those of all the
// slots, four rows at a time where the group allows it.
template <bool QUADS>
__global__ void __launch_bounds__(256) kv_weight_kernel(const Attend p, float* __restrict__ acc) {
    constexpr int kSlots = 4;
    pdl_wait();
    const int b = blockIdx.x / p.c.kv_heads, h = blockIdx.x % p.c.kv_heads;
    const Seq s = sequence<8, false>(p, b, nullptr);
    if (s.nq == 0) return;
    acc += (static_cast<int64_t>(b) * p.c.kv_heads + h) * p.S;
    for (int64_t s0 = static_cast<int64_t>(blockIdx.y) * (256 * kSlots) + threadIdx.x; s0 - threadIdx.x < s.n;
         s0 += static_cast<int64_t>(gridDim.y) * (256 * kSlots)) {
        float sum[kSlots], old[kSlots];
#pragma unroll
        for (int u = 0; u < kSlots; ++u) {
            sum[u] = 0.0f;
            if (s0 + u * 256 < s.n) old[u] = acc[s0 + u * 256];
        }
        for (int i = 0; i < s.nq; ++i) {
            const int64_t tk = s.first + i;
            const int end = visible(s.n, s.nq, i);
            const float* sc = p.scores + ((tk * p.c.kv_heads + h) * p.S + s0) * p.group;
            const float* ls = p.lse + tk * p.q_heads + h * p.group;
            if constexpr (QUADS) {
                for (int g = 0; g < p.group; g += 8) {   // a 32-byte sector at a time where the group fills it
                    float4 x[kSlots][2];
                    const bool two = g + 4 < p.group;
#pragma unroll
                    for (int u = 0; u < kSlots; ++u)
                        if (s0 + u * 256 < end) {
                            const float4* at = reinterpret_cast<const float4*>(sc + static_cast<int64_t>(u) * 256 * p.group + g);
                            x[u][0] = at[0];
                            if (two) x[u][1] = at[1];
                        }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        if (q && !two) break;
                        const float* l = ls + g + 4 * q;
                        const float l0 = l[0] * kLog2e, l1 = l[1] * kLog2e, l2 = l[2] * kLog2e, l3 = l[3] * kLog2e;
#pragma unroll
                        for (int u = 0; u < kSlots; ++u)
                            if (s0 + u * 256 < end)
                                sum[u] += ex2(x[u][q].x - l0) + ex2(x[u][q].y - l1) + (ex2(x[u][q].z - l2) + ex2(x[u][q].w - l3));
                    }
                }
            } else {
                for (int g = 0; g < p.group; ++g) {
                    const float l0 = ls[g] * kLog2e;
#pragma unroll
                    for (int u = 0; u < kSlots; ++u)
                        if (s0 + u * 256 < end) sum[u] += ex2(sc[static_cast<int64_t>(u) * 256 * p.group + g] - l0);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kSlots; ++u)
            if (s0 + u * 256 < s.n && KQ_IN_RANGE(s0 + u * 256, p.S)) acc[s0 + u * 256] = old[u] + sum[u];
    }
}

int64_t most_items(int64_t tokens, int64_t batch, int64_t group, int64_t kv_heads, int64_t rows) {
    return (tokens * group / rows + std::min(batch, tokens)) * kv_heads;
}

template <typename T, int D, int NT, bool WINDOW>
kq_status run_attend(Attend& p, cudaStream_t stream) {
    using Sh = Shape<T, D, NT>;
    p.most_items = most_items(p.tokens, p.c.batch, p.group, p.c.kv_heads, Sh::kRows);
    static std::atomic<uint64_t> done{0};
    KQ_TRY(once_per_device(done, [] {
        KQ_CUDA(cudaFuncSetAttribute(kv_attend_kernel<T, D, NT, WINDOW>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     static_cast<int>(Sh::kSmem)));
        return KQ_OK;
    }));
    const int grid = std::min(kMaxRows / Sh::kRows, num_sms() * Sh::kCtas * kWarps) / kWarps;
    KQ_CUDA(launch_after(kv_attend_kernel<T, D, NT, WINDOW>, dim3(grid), dim3(kThreads), Sh::kSmem, stream, p));
    count_launch();
    // a sequence has ceil(queries group / rows) items a head: at most this many, and few of them have many
    // results each, with a block for each column to go through them
    const int64_t items = p.most_items;
    const bool few = items * 32 < static_cast<int64_t>(grid) * kWarps;
    KQ_CUDA(launch_after(kv_combine_kernel<T, D, NT>, dim3(static_cast<unsigned>(items), few ? Sh::kRows : NT), dim3(256), 0, stream, p));
    count_launch();
    return KQ_OK;
}

size_t al256(size_t b) { return (b + 255) & ~static_cast<size_t>(255); }
size_t part_bytes(int64_t dim) { return al256(2ull * kMaxRows * (dim + 2) * sizeof(float)); }
size_t joint_bytes(int64_t T, int64_t q_heads) { return al256(256 + 2ull * T * q_heads * sizeof(Joint)); }   // items: at most two a row

}  // namespace

KQ_DEBUG_UNIT(kv_attend)
}  // namespace kq

using namespace kq;

extern "C" size_t kq_kv_attend_workspace(int64_t T, int64_t q_heads, int64_t kv_heads, int64_t dim, int64_t S) {
    if (T < 1 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || dim < 1 || S < 0) return 0;
    return joint_bytes(T, q_heads) + part_bytes(dim) + al256(static_cast<size_t>(T) * q_heads * sizeof(float)) +
           static_cast<size_t>(T) * q_heads * S * sizeof(float);
}

namespace {
// Both calls; window 0: all slots.
kq_status attend(const char* who, const kq_kv_cache* cache, const void* q, int dtype, int64_t T, int64_t q_heads,
                 int64_t q_token_stride, int64_t q_head_stride, const int32_t* start, const int32_t* lens, float scale,
                 int64_t window, int64_t sink, void* out, float* lse, float* acc, int64_t S, int* info, void* ws, size_t ws_bytes,
                 kq_stream_t stream_) {
    KvView c;
    KQ_TRY(kv_view(cache, who, &c));
    if (dtype != KQ_BF16 && dtype != KQ_F32) {
        set_error("%s: dtype must be KQ_BF16 or KQ_F32", who);
        return KQ_ERR_UNSUPPORTED;
    }
    const uintptr_t es = dtype == KQ_BF16 ? 2 : 4;
    if (T < 0 || T > 0x7fffffffll || q_heads < 1 || q_heads > 0x7fffffffll || q_heads % c.kv_heads || !start || !lens ||
        (T > 0 && (!q || !out)) || (acc && S < 1) || S > 0x7fffffffll || !(scale - scale == 0.0f) ||
        T * q_heads > 0x3fffffffll ||
        ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & (es - 1))) {
        set_error("%s: q, out, start, lens must not be NULL, q_heads a multiple of kv_heads, T q_heads < 2^30, "
                  "scale finite, S >= 1 with acc", who);
        return KQ_ERR_INVALID_ARG;
    }
    if (T == 0) return KQ_OK;
    const size_t need = kq_kv_attend_workspace(T, q_heads, c.kv_heads, c.dim, acc ? S : 0);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u)) {
        set_error("%s: workspace must be 256-byte aligned and hold %zu bytes", who, need);
        return KQ_ERR_WORKSPACE;
    }
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    uint8_t* w = static_cast<uint8_t*>(ws);
    Attend p;
    p.c = c;
    p.q = q;
    p.tokens = T;
    p.q_token = q_token_stride;
    p.q_head = q_head_stride;
    p.q_heads = static_cast<int32_t>(q_heads);
    p.group = static_cast<int32_t>(q_heads / c.kv_heads);
    p.q_vec = !(reinterpret_cast<uintptr_t>(q) & 15u) && !((q_token_stride * es) & 15u) && !((q_head_stride * es) & 15u);
    p.start = start;
    p.lens = lens;
    p.scale = scale;
    p.out = out;
    p.items = reinterpret_cast<int64_t*>(w);
    p.joint = reinterpret_cast<Joint*>(w + 256);
    p.part = reinterpret_cast<float*>(w + joint_bytes(T, q_heads));
    float* sums = reinterpret_cast<float*>(w + joint_bytes(T, q_heads) + part_bytes(c.dim));
    p.lse = lse ? lse : acc ? sums : nullptr;
    p.scores = acc ? sums + al256(static_cast<size_t>(T) * q_heads * sizeof(float)) / sizeof(float) : nullptr;
    p.S = S;
    p.cap = acc ? std::min(S, kv_capacity(c)) : kv_capacity(c);
    p.info = info;
    // Up to 8 rows of a key/value head fill one accumulator tile; more take two, so that the cache is
    // read half as often (a tensor-core column costs the same whether a row fills it or not).
    const bool wide = p.group > 8 || T > c.batch;
    constexpr int64_t kFar = 0x7fffffff;   // no sequence is longer
    p.window = static_cast<int32_t>(std::min(window, kFar));
    p.sink = static_cast<int32_t>(std::min(sink, kFar));
    // a window that no sequence can outgrow is none
    const bool limited = window > 0 && window < kv_capacity(c);
    auto pick = [&](auto t, auto d, auto n) {
        using E = decltype(t);
        return limited ? run_attend<E, decltype(d)::value, decltype(n)::value, true>(p, stream)
                       : run_attend<E, decltype(d)::value, decltype(n)::value, false>(p, stream);
    };
    auto pick_rows = [&](auto t, auto d) {
        return wide ? pick(t, d, std::integral_constant<int, 2>()) : pick(t, d, std::integral_constant<int, 1>());
    };
    auto pick_dim = [&](auto t) {
        return c.dim == 128 ? pick_rows(t, std::integral_constant<int, 128>()) : pick_rows(t, std::integral_constant<int, 64>());
    };
    const kq_status st = dtype == KQ_BF16 ? pick_dim(__nv_bfloat16()) : pick_dim(float());
    KQ_TRY(st);
    if (acc) {
        // enough blocks for two rounds of a full GPU, each going through its slots in steps of 1024
        const int64_t heads = static_cast<int64_t>(c.batch) * c.kv_heads;
        const dim3 wg(static_cast<unsigned>(heads),
                      static_cast<unsigned>(std::min<int64_t>(cdiv(p.cap, 1024), std::max<int64_t>(1, cdiv(num_sms() * 16, heads)))));
        KQ_CUDA(p.group % 4 ? launch_after(kv_weight_kernel<false>, wg, dim3(256), 0, stream, p, acc)
                            : launch_after(kv_weight_kernel<true>, wg, dim3(256), 0, stream, p, acc));
        count_launch();
    }
    return KQ_OK;
}
}  // namespace

extern "C" kq_status kq_kv_attend(const kq_kv_cache* cache, const void* q, int dtype, int64_t T, int64_t q_heads,
                                  int64_t q_token_stride, int64_t q_head_stride, const int32_t* start,
                                  const int32_t* lens, float scale, void* out, float* lse, float* acc, int64_t S, int* info,
                                  void* ws, size_t ws_bytes, kq_stream_t stream) {
    return attend("kq_kv_attend", cache, q, dtype, T, q_heads, q_token_stride, q_head_stride, start, lens, scale, 0, 0, out, lse,
                  acc, S, info, ws, ws_bytes, stream);
}

extern "C" kq_status kq_kv_attend_window(const kq_kv_cache* cache, const void* q, int dtype, int64_t T, int64_t q_heads,
                                         int64_t q_token_stride, int64_t q_head_stride, const int32_t* start,
                                         const int32_t* lens, float scale, int64_t window, int64_t sink, void* out, float* lse,
                                         int* info, void* ws, size_t ws_bytes, kq_stream_t stream) {
    if (window < 1 || sink < 0) {
        set_error("kq_kv_attend_window: window >= 1 and sink >= 0 needed");
        return KQ_ERR_INVALID_ARG;
    }
    return attend("kq_kv_attend_window", cache, q, dtype, T, q_heads, q_token_stride, q_head_stride, start, lens, scale, window,
                  sink, out, lse, nullptr, 0, info, ws, ws_bytes, stream);
}
