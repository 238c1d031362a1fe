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

// One CTA per row (t, h): each warp takes every fourth key with its own running
// maximum and sum, and the four are joined at the end.
template <typename T>
__global__ void __launch_bounds__(32 * kWarps) k_attend_rows(const __grid_constant__ Args<T> a) {
    const AttendJob &j = a.j;
    const KvView &kv = a.kv;
    __shared__ float s_m[kWarps], s_l[kWarps], s_o[kWarps][32 * kPer];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int t = blockIdx.x / j.Hq, h = blockIdx.x % j.Hq, hk = h / (j.Hq / kv.heads);
    const int b = kv.seq(t), len = kv.len(b);
    if (kv.news(b) * (j.Hq / kv.heads) <= kFewRows) return;
    int lo, hi;
    reach(j, len, len - kv.news(b) + t - kv.first(b), lo, hi);
    float q[kPer], o[kPer] = {}, m = -INFINITY, l = 0.0f;
    load_row<T>(static_cast<const char *>(j.q) + t * j.q_token + h * j.q_head, kv.dim, lane, q);
#pragma unroll
    for (int i = 0; i < kPer; ++i) q[i] *= j.scale;
    for (int k = lo + warp; k < hi; k += kWarps) {
        int page, slot;
        if (!kv.place(b, k, page, slot)) continue;
        float x[kPer];
        load_row<T>(kv.K + page * kv.k_page + slot * kv.k_slot + hk * kv.k_head, kv.dim, lane, x);
        const float s = dot(q, x), mn = fmaxf(m, s);
        const float old = m == -INFINITY ? 0.0f : expf(m - mn), p = expf(s - mn);
        load_row<T>(kv.V + page * kv.v_page + slot * kv.v_slot + hk * kv.v_head, kv.dim, lane, x);
        l = l * old + p;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] = o[i] * old + p * x[i];
        m = mn;
    }
    if (lane == 0) s_m[warp] = m, s_l[warp] = l;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s_o[warp][lane + 32 * i] = o[i];
    __syncthreads();
    float mm = -INFINITY, ll = 0.0f;
    for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, s_m[w]);
    for (int w = 0; w < kWarps; ++w) ll += s_m[w] == -INFINITY ? 0.0f : s_l[w] * expf(s_m[w] - mm);
    T *out = reinterpret_cast<T *>(static_cast<char *>(j.out) + t * j.o_token + h * j.o_head);
    for (int d = threadIdx.x; d < kv.dim; d += 32 * kWarps) {
        float v = 0.0f;
        for (int w = 0; w < kWarps; ++w)
            if (s_m[w] != -INFINITY) v += s_o[w][d] * expf(s_m[w] - mm);
        out[d] = from_f32<T>(ll > 0.0f ? v / ll : ll);
    }
    if (threadIdx.x == 0 && j.lse) j.lse[(int64_t)t * j.Hq + h] = mm + logf(ll);
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
        const cudaError_t e = stream_scratch(kScratchAttention, (size_t)kv.T * j.Hq * sizeof(float), s, &p);
        if (e != cudaSuccess) return e;
        a.j.lse = static_cast<float *>(p);
    }
    k_attend_rows<T><<<(unsigned)(kv.T * j.Hq), 32 * kWarps, 0, s>>>(a);
    cudaError_t e = counted_launch(cudaGetLastError());
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
