// Eviction from a paged cache by accumulated attention weight (pvmvmd_kv_evict).
//
// k_evict_select, a CTA per (sequence, head): the kept tokens' indexes, ascending.
// Masses map to integers of the same order; four passes of 8 bits find the value of
// the last one kept and how many equal ones stay, and a scan writes the list.
// k_evict_move, a CTA per (sequence, head): the rows of the list in order, some at a
// time.  A row never moves to a higher index, so what is written over has been read
// when every row of a step is read before any is written.
#include "attention.h"
#include "kv.cuh"

namespace pv {
namespace {

constexpr int kSelThreads = 512;
constexpr int kMoveThreads = 256;

struct EvictArgs {
    EvictJob j;
    KvView kv;
    int32_t *list;  // [B][heads][budget]
    int32_t *kept;  // [B]
};

// Order-preserving image of a mass; NaN below every number.
__device__ __forceinline__ uint32_t mass_key(float v) {
    if (v != v) return 0u;
    const uint32_t u = __float_as_uint(v + 0.0f);  // -0 and 0 are equal
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelThreads) k_evict_select(const __grid_constant__ EvictArgs a) {
    const KvView &kv = a.kv;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int len = kv.len(b), n = min(len, a.j.budget), fixed = min(a.j.recent, n);
    const int cand = len - fixed, want = n - fixed;
    int32_t *list = a.list + ((int64_t)b * kv.heads + h) * a.j.budget;
    if (h == 0 && tid == 0) a.kept[b] = n;
    if (n == len) {
        for (int i = tid; i < n; i += kSelThreads) list[i] = i;
        return;
    }
    for (int i = tid; i < fixed; i += kSelThreads) list[want + i] = cand + i;
    if (want == 0) return;
    auto key_at = [&](int i) {
        int page, slot;
        return kv.place(b, i, page, slot) ? mass_key(*kv.mass_at(page, slot, h)) : 0u;
    };
    __shared__ int hist[256], s_left;
    __shared__ uint32_t s_value;
    uint32_t value = 0, mask = 0;  // digits of the last kept one found so far
    int left = want;               // of the candidates that share them
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < cand; i += kSelThreads) {
            const uint32_t k = key_at(i);
            if ((k & mask) == value) atomicAdd(&hist[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int d = 255, above = 0;
            while (d > 0 && above + hist[d] < left) above += hist[d--];
            s_value = value | (uint32_t)d << shift;
            s_left = left - above;
        }
        __syncthreads();
        value = s_value;
        left = s_left;
        mask |= 255u << shift;
    }
    // kept: those above value, and the first `left` equal to it
    __shared__ int s_gt[kSelThreads / 32], s_eq[kSelThreads / 32];
    int gt0 = 0, eq0 = 0;
    for (int i0 = 0; i0 < cand; i0 += kSelThreads) {
        const int i = i0 + tid;
        const uint32_t k = i < cand ? key_at(i) : 0u;
        const unsigned gt = __ballot_sync(kFull, i < cand && k > value), eq = __ballot_sync(kFull, i < cand && k == value);
        if (lane == 0) s_gt[warp] = __popc(gt), s_eq[warp] = __popc(eq);
        __syncthreads();
        int g = gt0 + __popc(gt & lanemask_lt()), e = eq0 + __popc(eq & lanemask_lt());
        for (int w = 0; w < kSelThreads / 32; ++w) {
            if (w < warp) g += s_gt[w], e += s_eq[w];
            gt0 += s_gt[w], eq0 += s_eq[w];
        }
        if (i < cand && (k > value || (k == value && e < left))) list[g + min(e, left)] = i;
        __syncthreads();
    }
}

constexpr int kMoveChunks = 8;  // 16-byte chunks per thread and step

__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const __grid_constant__ EvictArgs a) {
    const KvView &kv = a.kv;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int n = a.kept[b], per_part = kv.dim / 8, per = 2 * per_part;
    const int32_t *list = a.list + ((int64_t)b * kv.heads + h) * a.j.budget;
    const int rows = kMoveThreads * kMoveChunks / per;
    for (int r0 = 0; r0 < n; r0 += rows) {
        uint4 x[kMoveChunks];
        char *to[kMoveChunks];
        const int m = min(rows, n - r0);
        // of a row, chunks of its key, then of its value
#pragma unroll
        for (int c = 0; c < kMoveChunks; ++c) {
            const int id = tid + c * kMoveThreads, r = id / per, part = id % per;
            to[c] = nullptr;
            if (r >= m) continue;
            const bool v = part >= per_part;
            const int64_t off = (int64_t)(v ? part - per_part : part) * 16;
            int sp, ss, dp;
            uint32_t q, ds;
            if (!kv.place(b, list[r0 + r], sp, ss)) continue;
            kv.ps.divmod((uint32_t)(r0 + r), q, ds);
            dp = a.j.new_table[b * a.j.new_stride + q];
            if (dp < 0 || dp >= kv.pages) continue;
            const char *src = (v ? kv.V + sp * kv.v_page + ss * kv.v_slot + h * kv.v_head
                                 : kv.K + sp * kv.k_page + ss * kv.k_slot + h * kv.k_head) + off;
            to[c] = (v ? kv.V + dp * kv.v_page + ds * kv.v_slot + h * kv.v_head
                       : kv.K + dp * kv.k_page + ds * kv.k_slot + h * kv.k_head) + off;
            x[c] = *reinterpret_cast<const uint4 *>(src);
        }
        float w = 0.0f, *wto = nullptr;
        if (tid < m) {
            int sp, ss, dp;
            uint32_t q, ds;
            kv.ps.divmod((uint32_t)(r0 + tid), q, ds);
            dp = a.j.new_table[b * a.j.new_stride + q];
            if (kv.place(b, list[r0 + tid], sp, ss) && dp >= 0 && dp < kv.pages) {
                w = *kv.mass_at(sp, ss, h);
                wto = kv.mass_at(dp, (int)ds, h);
            }
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < kMoveChunks; ++c)
            if (to[c]) *reinterpret_cast<uint4 *>(to[c]) = x[c];
        if (wto) *wto = w;
        __syncthreads();
    }
    if (h == 0 && tid == 0) a.j.new_lens[b] = n;
}

}  // namespace

cudaError_t launch_evict(const EvictJob &j, const KvView &kv, cudaStream_t s) {
    EvictArgs a{j, kv, nullptr, nullptr};
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d;
    if (a.j.budget > room) a.j.budget = (int)room;  // no sequence is longer
    void *p = nullptr;
    const size_t lists = (size_t)kv.B * kv.heads * a.j.budget;
    const cudaError_t e = stream_scratch(kScratchAttention, (lists + kv.B) * sizeof(int32_t), s, &p);
    if (e != cudaSuccess) return e;
    a.list = static_cast<int32_t *>(p);
    a.kept = a.list + lists;
    const dim3 grid((unsigned)kv.heads, (unsigned)kv.B);
    k_evict_select<<<grid, kSelThreads, 0, s>>>(a);
    const cudaError_t e1 = counted_launch(cudaGetLastError());
    if (e1 != cudaSuccess) return e1;
    k_evict_move<<<grid, kMoveThreads, 0, s>>>(a);
    return counted_launch(cudaGetLastError());
}

}  // namespace pv
