// The paged cache as the kernels of the client's attention see it
// (pvmvmd_kv_pool and pvmvmd_kv_batch of include/pvmvmd.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>
#include <cstdint>

#include "common.cuh"

namespace pv {

// n / d for 0 <= n < 2^31 (Granlund and Montgomery, PLDI 1994, Fig. 4.1): with
// 2^shift >= d and mul = floor(2^32 (2^shift - d) / d) + 1 the quotient is
// (hi(n mul) + n) >> shift.
struct FastDiv {
    uint32_t d, mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t div) : d(div), shift(0) {
        while (((uint64_t)1 << shift) < d) ++shift;
        mul = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ void divmod(uint32_t n, uint32_t &q, uint32_t &r) const {
        q = (__umulhi(n, mul) + n) >> shift;
        r = n - q * d;
    }
};

struct KvView {
    char *K, *V;
    float *mass;
    int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;  // bytes
    int pages, heads, dim;
    FastDiv ps;  // page size
    const int32_t *table, *lens, *cu;
    int64_t table_stride;
    int B, T, max_pages, max_new;

    // cached tokens of sequence b, no more than its table has room for
    __device__ __forceinline__ int len(int b) const {
        const int64_t room = (int64_t)max_pages * ps.d;
        const int l = max(lens[b], 0);
        return room < l ? (int)room : l;
    }
    // first row and number of the new tokens of sequence b: rows of the T there are, and
    // no more than scratch is made for, whatever cu holds
    __device__ __forceinline__ int first(int b) const { return cu ? min(max(cu[b], 0), T) : b; }
    __device__ __forceinline__ int news(int b) const {
        return cu ? min(max(min(cu[b + 1], T) - first(b), 0), max_new) : 1;
    }
    // the sequence of row t
    __device__ __forceinline__ int seq(int t) const {
        if (!cu) return t;
        int lo = 0, hi = B;  // cu[lo] <= t < cu[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cu[mid] <= t)
                lo = mid;
            else
                hi = mid;
        }
        return lo;
    }
    // the cache index of new token t of sequence b = seq(t); negative in front of the
    // sequence's start, and the least one of a row that is no token of it
    __device__ __forceinline__ int index(int b, int t) const {
        const int n = news(b), i = t - first(b);
        return i >= 0 && i < n ? len(b) - n + i : INT_MIN;
    }
    // page and slot of cache index i of sequence b; false where there is none
    __device__ __forceinline__ bool place(int b, int i, int &page, int &slot) const {
        uint32_t p, o;
        ps.divmod((uint32_t)i, p, o);
        page = table[b * table_stride + p];
        slot = (int)o;
        return page >= 0 && page < pages;
    }
    __device__ __forceinline__ float *mass_at(int page, int slot, int h) const {
        return mass + ((int64_t)page * heads + h) * ps.d + slot;
    }
};

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
// a field element as the centred integer it stands for
template <>
__device__ __forceinline__ float to_f32(uint32_t v) { return (float)(v > kHalfQ ? (int)(v - kQ) : (int)v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

}  // namespace pv
