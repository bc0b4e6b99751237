// laq_paged.cuh -- what the paged-cache kernels share (not installed): the two 16-bit types, the
// cache's description as the kernels take it, and the host checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "laq.h"

namespace laq {

constexpr int kPagedDim = 128;  // D

// laq_paged_kv, checked, as a kernel parameter.  page_size = 1 << page_bits.
struct PagedKv {
    uint16_t *k, *v;
    const int32_t *table, *q_start, *kv_len;
    int64_t pages, page_stride, head_stride, token_stride, table_stride;
    int32_t batch, max_tokens, page_bits, Hkv;
};

// The checks of a laq_paged_kv that every call makes, and its kernel form.  T rows (for the sizes).
laq_status paged_kv(const laq_paged_kv* kv, int64_t T, int32_t Hq, PagedKv* out);

namespace {

template <bool BF>
struct Half16;
template <>
struct Half16<false> {
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return __half22float2(*reinterpret_cast<const __half2*>(&w));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <>
struct Half16<true> {
    static __device__ __forceinline__ float2 unpack(uint32_t w) {
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

// The request whose rows include row t: the number of entries of q_start[1 .. batch] that are <= t
// (nondecreasing), by the whole warp: every step reads 32 of them and keeps a 32nd of what is left.
__device__ __forceinline__ int request_of(const int32_t* __restrict__ q_start, int batch, int t) {
    const int lane = threadIdx.x & 31;
    int lo = 0, n = batch;  // the answer is in [lo, lo + n]
    while (n > 0) {
        const int step = (n + 31) / 32;
        const int at = lo + (lane + 1) * step;  // entry `at` counts all of (lo, at]
        const bool below = at <= lo + n && q_start[at] <= t;
        const int c = __popc(__ballot_sync(0xffffffffu, below));
        const int left = n - c * step;
        lo += c * step;
        n = min(left, step - 1);
    }
    return lo;
}

}  // namespace
}  // namespace laq
