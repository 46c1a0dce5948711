// The 4-bit key/value cache: layout, addressing and the device-side checks that its entry
// points share.
//
// data holds `pages` pages; a page holds, for each key/value head, page / 16 granules of 16
// tokens. A granule is one run of 16 (D + 8) bytes:
//     16 rows of D / 2 bytes   key codes (dim 2 j in the low half of byte j)
//     16 rows of D / 2 bytes   value codes
//     16 pairs of bf16         key (scale, offset)
//     16 pairs of bf16         value (scale, offset)
// so that the tokens of a tile, with everything needed to read them, are one contiguous run
// whose length and address are multiples of 16 bytes for every page size.
#pragma once

#include <cuda_bf16.h>

#include "kq_common.cuh"

namespace kq {

constexpr int kGranule = 16;   // tokens

struct KvView {
    uint8_t* data;
    const int32_t* table;   // [batch][table_ld] page numbers
    int64_t pages;
    int32_t page;           // tokens of a page
    int32_t kv_heads;
    int32_t dim;
    int32_t batch;
    int64_t table_ld;
};

__host__ __device__ __forceinline__ int64_t kv_head_bytes(const KvView& c) {
    return static_cast<int64_t>(c.page) * (c.dim + 8);
}
__host__ __device__ __forceinline__ int64_t kv_pool_bytes(const KvView& c) { return c.pages * c.kv_heads * kv_head_bytes(c); }
__host__ __device__ __forceinline__ int64_t kv_capacity(const KvView& c) { return c.table_ld * c.page; }

// The granule of slot `slot` (0 <= slot < capacity) of sequence b and head h, or nullptr when
// the table names a page that the pool does not have.
__device__ __forceinline__ uint8_t* kv_granule(const KvView& c, int b, int h, int64_t slot_) {
    const uint32_t slot = static_cast<uint32_t>(slot_), pg = slot / static_cast<uint32_t>(c.page);
    const int64_t p = c.table[static_cast<int64_t>(b) * c.table_ld + pg];
    if (p < 0 || p >= c.pages) return nullptr;
    return c.data + (p * c.kv_heads + h) * kv_head_bytes(c) +
           (slot - pg * static_cast<uint32_t>(c.page)) / kGranule * (kGranule * (c.dim + 8));
}
// Byte offsets in a granule: the code row and the (scale, offset) pair of its token t; which = 0
// for the key, 1 for the value.
__device__ __forceinline__ int kv_code_at(int dim, int which, int t) { return (which * kGranule + t) * (dim / 2); }
__device__ __forceinline__ int kv_param_at(int dim, int which, int t) {
    return kGranule * dim + (which * kGranule + t) * 4;
}
__device__ __forceinline__ float kv_scale(uint32_t param) { return __uint_as_float(param << 16); }
__device__ __forceinline__ float kv_offset(uint32_t param) { return __uint_as_float(param & 0xFFFF0000u); }

// The sequence b whose tokens start[b] .. start[b + 1] - 1 hold token i, or -1. start is not
// trusted: the result is checked against both ends.
__device__ __forceinline__ int kv_sequence_of(const int32_t* __restrict__ start, int batch, int64_t i) {
    int lo = 0, hi = batch;   // the first b with start[b + 1] > i
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (start[mid + 1] > i) hi = mid;
        else lo = mid + 1;
    }
    return lo < batch && start[lo] <= i && i < start[lo + 1] ? lo : -1;
}

// The same by a whole warp, 32 sequences at a look.
__device__ __forceinline__ int kv_sequence_of_warp(const int32_t* __restrict__ start, int batch, int64_t i) {
    const int lane = threadIdx.x & 31;
    int lo = 0, len = batch;
    while (len > 0) {
        const int step = (len + 31) >> 5, end = min((lane + 1) * step, len);   // lane's sequences end before lo + end
        const bool before = lane * step < len && start[lo + end] <= i;
        const int n = __popc(__ballot_sync(0xffffffffu, before)) * step;
        lo += min(n, len);
        if (step == 1) break;
        len = min(step, len - n);
    }
    return lo < batch && start[lo] <= i && i < start[lo + 1] ? lo : -1;
}

// The length of sequence b, brought into 0 .. most; a length outside is recorded in info.
__device__ __forceinline__ int64_t kv_length(const int32_t* __restrict__ lens, int b, int64_t most, int* info) {
    const int64_t n = lens[b];
    if (n >= 0 && n <= most) return n;
    record_error(info, -KQ_ERR_INVALID_ARG);
    return n < 0 ? 0 : most;
}

// Host side: whether an output of n integers shares memory with m integers that blocks still read while it is written.
inline bool kv_overlap(const int32_t* out, int64_t n, const int32_t* in, int64_t m) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(out), b = reinterpret_cast<uintptr_t>(in);
    return out && in && a < b + static_cast<uintptr_t>(m) * sizeof(int32_t) && b < a + static_cast<uintptr_t>(n) * sizeof(int32_t);
}

// Host side: checks a cache description and makes the kernels' view of it.
kq_status kv_view(const kq_kv_cache* c, const char* who, KvView* v);

}  // namespace kq
