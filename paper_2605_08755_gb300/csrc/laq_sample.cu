// laq_sample.cu -- the next token of each row of logits: temperature, top-k, top-p and min-p, and the
// choice by a given random number.
//
// Weights are whole numbers (2^40 for the maximum), so that every sum is exact and no result depends
// on how a sum is split; logits map to 32-bit keys of the same order.  What top-k and top-p keep is a
// prefix of the order (key descending, index ascending): all keys above some key, and the first few
// of that key.  The prefix is found digit by digit of the key (a histogram of counts and weights per
// digit), the token by prefix sums of the kept weights in the order of the index.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "laq.h"
#include "laq_device.cuh"

namespace laq {
namespace {

constexpr int kThreads = 1024;
typedef unsigned long long u64;

template <int DT>
__device__ __forceinline__ float load_logit(const void* row, int64_t i) {
    float x;
    if (DT == LAQ_F32) x = static_cast<const float*>(row)[i];
    else if (DT == LAQ_F16) x = __half2float(static_cast<const __half*>(row)[i]);
    else x = __bfloat162float(static_cast<const __nv_bfloat16*>(row)[i]);
    return isnan(x) ? -INFINITY : x + 0.f;  // (+ 0: the two zeros are one value)
}
// order-preserving key
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ u64 weight(float x, float top, float t) {
    return x == top ? (u64)1 << 40 : (u64)(expf((x - top) / t) * 0x1p40f);
}
// floor(mass * f / 2^24), mass < 2^63, f <= 2^24
__device__ __forceinline__ u64 part(u64 mass, uint32_t f) {
    return (mass >> 24) * f + (((mass & 0xffffffu) * f) >> 24);
}

// What is kept: keys above `key`, and the first `count` (by index) of those equal to it.
struct Cut {
    uint32_t key;
    u64 count;
};

struct SampleParams {
    const void* logits;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* out;
    float* p_out;
    int64_t row_stride;
    int V;
};

template <typename T>
__device__ __forceinline__ T block_sum(T v, T* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    T s = 0;
    for (int k = 0; k < kThreads / 32; ++k) s += red[k];
    return s;
}

template <int DT>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams p) {
    pdl_launch_dependents();
    pdl_wait();
    __shared__ u64 red[32], hist_w[256];
    __shared__ uint32_t hist_n[256];
    __shared__ u64 pick[4];
    __shared__ float fred[32];
    const int m = blockIdx.x, V = p.V, tid = threadIdx.x;
    const size_t size = DT == LAQ_F32 ? 4 : 2;
    const void* row = static_cast<const char*>(p.logits) + (size_t)m * p.row_stride * size;
    float top = -INFINITY;
    for (int i = tid; i < V; i += kThreads) top = fmaxf(top, load_logit<DT>(row, i));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if ((tid & 31) == 0) fred[tid >> 5] = top;
    __syncthreads();
    for (int k = 0; k < 32; ++k) top = fmaxf(top, fred[k]);
    if (top == -INFINITY) {
        if (tid == 0) {
            p.out[m] = 0;
            if (p.p_out) p.p_out[m] = 0.f;
        }
        return;
    }
    float t = p.temperature ? p.temperature[m] : 1.f;
    const bool greedy = !(t > 0.f);
    int64_t k = p.top_k ? p.top_k[m] : 0;
    if (k <= 0 || k > V) k = V;
    if (greedy) {
        k = 1;
        t = 1.f;
    }
    const float fp = p.top_p ? p.top_p[m] : 1.f, fm = p.min_p ? p.min_p[m] : 0.f;
    const bool use_p = fp < 1.f && !greedy;
    const uint32_t pf = use_p ? (uint32_t)(fmaxf(fp, 0.f) * 0x1p24f) : 0u;
    const u64 floor_w = fm > 0.f && !greedy ? (u64)(fminf(fm, 1.f) * 0x1p40f) : 0;
    const float u = p.u[m];
    const uint32_t uf = u > 0.f ? min((uint32_t)(fminf(u, 1.f) * 0x1p24f), 0xffffffu) : 0u;

    // The shortest prefix of the order, within `in`, of `need` elements or (BY_MASS) of a weight of at
    // least `need`; *mass: the prefix's weight.
    auto find = [&](bool by_mass, u64 need, u64* mass) {
        uint32_t prefix = 0;
        u64 above_w = 0;
        Cut cut = {0u, 0};
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist_n[tid] = 0, hist_w[tid] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += kThreads) {
                const float x = load_logit<DT>(row, i);
                const uint32_t key = key_of(x);
                if (shift < 24 && (key >> (shift + 8)) != (prefix >> (shift + 8))) continue;
                atomicAdd(&hist_n[(key >> shift) & 255], 1u);
                atomicAdd(&hist_w[(key >> shift) & 255], weight(x, top, t));
            }
            __syncthreads();
            if (tid == 0) {
                int d = 255;
                u64 w = above_w, left = need;
                for (; d > 0; --d) {
                    const u64 a = by_mass ? hist_w[d] : hist_n[d];
                    if (a >= left && hist_n[d]) break;
                    left -= min(a, left);
                    w += hist_w[d];
                }
                pick[0] = d;
                pick[1] = left;
                pick[2] = w;
                pick[3] = hist_n[d];
            }
            __syncthreads();
            prefix |= (uint32_t)pick[0] << shift;
            need = pick[1];
            above_w = pick[2];
            cut.count = pick[3];
            __syncthreads();
        }
        cut.key = prefix;
        // elements of the last key: all of one weight
        const uint32_t b = (prefix & 0x80000000u) ? prefix ^ 0x80000000u : ~prefix;
        const u64 w = weight(__uint_as_float(b), top, t);
        if (by_mass) cut.count = w ? min(cut.count, max((u64)1, (need + w - 1) / w)) : cut.count;
        else cut.count = need;
        *mass = above_w + cut.count * w;
        return cut;
    };
    u64 mass = 0;
    Cut cut = {0u, 0x7fffffff};
    bool cut_on = false;
    if (k < V) {
        cut = find(false, (u64)k, &mass);
        cut_on = true;
    }
    if (use_p) {
        if (!cut_on) {
            u64 s = 0;
            for (int i = tid; i < V; i += kThreads) s += weight(load_logit<DT>(row, i), top, t);
            mass = block_sum(s, red);
        }
        cut = find(true, max((u64)1, part(mass, pf)), &mass);
        cut_on = true;
    }
    // kept weights in the order of the index: each thread a run of indices
    const int per = (V + kThreads - 1) / kThreads, i0 = min(V, tid * per), i1 = min(V, i0 + per);
    auto scan = [&](u64 v, u64* total) {  // exclusive prefix over the block
        u64 s = v;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const u64 y = __shfl_up_sync(0xffffffffu, s, o);
            if ((tid & 31) >= o) s += y;
        }
        __syncthreads();
        if ((tid & 31) == 31) red[tid >> 5] = s;
        __syncthreads();
        u64 before = 0, all = 0;
        for (int j = 0; j < 32; ++j) {
            if (j < (tid >> 5)) before += red[j];
            all += red[j];
        }
        *total = all;
        return before + s - v;
    };
    u64 eq = 0, all;
    if (cut_on)
        for (int i = i0; i < i1; ++i) eq += key_of(load_logit<DT>(row, i)) == cut.key;
    const u64 eq0 = scan(eq, &all);
    auto kept = [&](int i, u64& seen) {
        const float x = load_logit<DT>(row, i);
        const uint32_t key = key_of(x);
        bool on = !cut_on || key > cut.key;
        if (cut_on && key == cut.key) on = seen++ < cut.count;
        const u64 w = on ? weight(x, top, t) : 0;
        return w >= floor_w ? w : 0;
    };
    u64 s = 0, seen = eq0, total;
    for (int i = i0; i < i1; ++i) s += kept(i, seen);
    u64 before = scan(s, &total);
    const u64 target = part(total, uf);
    if (before <= target && target < before + s) {
        seen = eq0;
        for (int i = i0; i < i1; ++i) {
            const u64 w = kept(i, seen);
            before += w;
            if (before > target) {
                p.out[m] = i;
                if (p.p_out) p.p_out[m] = (float)w / (float)total;
                break;
            }
        }
    }
}

template <int DT>
laq_status launch_sample(const SampleParams& p, int64_t M, void* stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)M);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sample_kernel<DT>, p) == cudaSuccess ? LAQ_OK : LAQ_ERR_CUDA;
}

}  // namespace
}  // namespace laq

using namespace laq;

extern "C" laq_status laq_sample(const void* logits, int32_t dtype, int64_t M, int64_t V,
                                 int64_t row_stride, const float* temperature,
                                 const int32_t* top_k, const float* top_p, const float* min_p,
                                 const float* u, int32_t* out, float* p_out, void* stream) {
    if (dtype != LAQ_F16 && dtype != LAQ_BF16 && dtype != LAQ_F32) return LAQ_ERR_CONFIG;
    if (M < 0 || M > 65535 || V < 1 || V > (int64_t)1 << 22 || row_stride < V ||
        row_stride > (int64_t)1 << 40)
        return LAQ_ERR_SHAPE;
    if (M == 0) return LAQ_OK;
    if (!logits || !u || !out) return LAQ_ERR_NULL;
    if (((uintptr_t)logits & (dtype == LAQ_F32 ? 3u : 1u)) ||
        (((uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p |
          (uintptr_t)u | (uintptr_t)out | (uintptr_t)p_out) & 3u))
        return LAQ_ERR_ALIGN;
    const SampleParams p = {logits, temperature, top_p, min_p, u, top_k, out, p_out, row_stride,
                            (int)V};
    if (dtype == LAQ_F32) return launch_sample<LAQ_F32>(p, M, stream);
    if (dtype == LAQ_BF16) return launch_sample<LAQ_BF16>(p, M, stream);
    return launch_sample<LAQ_F16>(p, M, stream);
}
