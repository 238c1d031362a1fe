// Attention of new tokens over a paged cache (pvmvmd_paged_attention).
#include <cfloat>

#include "attention.h"
#include "kv.cuh"

namespace pv {
namespace {

constexpr int kWarps = 4;
constexpr int kPer = PVMVMD_MAX_HEAD / 32;  // values of a head per lane

template <typename T>
struct Args {
    AttendJob j;
    KvView kv;
};

template <typename T>
__device__ __forceinline__ void load_row(const char *row, int dim, int lane, float (&x)[kPer]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int d = lane + 32 * i;
        x[i] = d < dim ? to_f32(reinterpret_cast<const T *>(row)[d]) : 0.0f;
    }
}
__device__ __forceinline__ float dot(const float (&a)[kPer], const float (&b)[kPer]) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s += a[i] * b[i];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    return s;
}
// keys [lo, hi) that a row at cache index i sees
__device__ __forceinline__ void reach(const AttendJob &j, int len, int i, int &lo, int &hi) {
    hi = j.causal ? min(len, i + 1) : len;
    lo = j.window > 0 && i >= j.window ? i - j.window + 1 : 0;
    if (hi < 0) hi = 0;
}

// The mass of one key per warp: the rows that see it, in order.
template <typename T>
__global__ void __launch_bounds__(32 * kWarps) k_mass_keys(const __grid_constant__ Args<T> a, const float *lse) {
    const AttendJob &j = a.j;
    const KvView &kv = a.kv;
    const int lane = threadIdx.x & 31;
    const int b = blockIdx.z, hk = blockIdx.y, k = blockIdx.x * kWarps + (threadIdx.x >> 5), len = kv.len(b);
    int page, slot;
    if (k >= len || !kv.place(b, k, page, slot)) return;
    const int G = j.Hq / kv.heads, t0 = kv.first(b), n = kv.news(b);
    if (n * G <= kFewRows) return;
    float x[kPer], q[kPer], sum = 0.0f;
    load_row<T>(kv.K + page * kv.k_page + slot * kv.k_slot + hk * kv.k_head, kv.dim, lane, x);
    for (int t = 0; t < n; ++t) {
        int lo, hi;
        reach(j, len, len - n + t, lo, hi);
        if (k < lo || k >= hi) continue;
        for (int g = 0; g < G; ++g) {
            const int h = hk * G + g;
            load_row<T>(static_cast<const char *>(j.q) + (t0 + t) * j.q_token + h * j.q_head, kv.dim, lane, q);
#pragma unroll
            for (int i = 0; i < kPer; ++i) q[i] *= j.scale;
            sum += expf(dot(q, x) - lse[(int64_t)(t0 + t) * j.Hq + h]);
        }
    }
    if (lane == 0) *kv.mass_at(page, slot, hk) += sum;
}

template <typename T>
cudaError_t attend(const AttendJob &j, const KvView &kv, cudaStream_t s) {
    Args<T> a{j, kv};
    if (j.accumulate && !j.lse) {
        void *p = nullptr;
        const cudaError_t e = stream_scratch(kScratchLse, (size_t)kv.T * j.Hq * sizeof(float), s, &p);
        if (e != cudaSuccess) return e;
        a.j.lse = static_cast<float *>(p);
    }
    cudaError_t e = launch_attention_chunk(a.j, kv, s);
    if (e != cudaSuccess || !j.accumulate) return e;
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d;
    const dim3 grid((unsigned)((room + kWarps - 1) / kWarps), (unsigned)kv.heads, (unsigned)kv.B);
    k_mass_keys<T><<<grid, 32 * kWarps, 0, s>>>(a, a.j.lse);
    return counted_launch(cudaGetLastError());
}

}  // namespace

cudaError_t launch_attention(const AttendJob &j, const KvView &kv, cudaStream_t s) {
    const int G = j.Hq / kv.heads;
    if (G <= kFewRows) {
        const cudaError_t e = launch_attention_few(j, kv, s);
        if (e != cudaSuccess || j.max_new <= kFewRows / G) return e;
    }
    return j.type == PVMVMD_BF16 ? attend<__nv_bfloat16>(j, kv, s) : attend<__half>(j, kv, s);
}

}  // namespace pv
