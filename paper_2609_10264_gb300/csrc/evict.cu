// Eviction from a paged cache by accumulated attention weight (pvmvmd_kv_evict).
//
// k_evict_select, a CTA per (sequence, head): the kept tokens' indexes, ascending.
// Masses map to integers of the same order, and the value of the last one kept is
// found two bits at a time: three counts of the keys not below a bound.  Keys stay
// in registers (up to 32768 of them; longer sequences are read again for each of
// four passes of 8 bits).  A scan over the counts of every warp's keys then gives
// each kept one its place.
//
// k_evict_move: the rows of a list, 16 KiB of keys and as many of values a CTA.  A row
// never moves to a higher index, so in place the rows that lie where a CTA writes are
// its own or those of CTAs before it: it reports its rows read and waits for their
// reports before it writes.  Blocks start in the order of their index (as the other
// kernels that chain blocks rest on); the wait is bounded.
#include "attention.cuh"

namespace pv {
namespace {

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kSelPer = 64;   // keys per thread in registers
constexpr int kMoveThreads = 256;
constexpr int kMoveChunks = 8;  // 16-byte chunks per thread

struct EvictArgs {
    EvictJob j;
    KvView kv;
    int32_t *list;    // [B][heads][budget]
    int32_t *kept;    // [B]
    uint32_t *loaded; // [B][heads][chunks]: rows read
    int rows, chunks; // per CTA of the move, per list
    uint32_t *err;
};

// Order-preserving image of a mass; NaN below every number.
__device__ __forceinline__ uint32_t mass_key(float v) {
    if (v != v) return 0u;
    const uint32_t u = __float_as_uint(v + 0.0f);  // -0 and 0 are equal
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint32_t key_at(const KvView &kv, int b, int h, int i) {
    int page, slot;
    return kv.place(b, i, page, slot) ? mass_key(*kv.mass_at(page, slot, h)) : 0u;
}

// The largest value of which at least `want` of `cand` keys are not below, and how
// many of those equal to it are among the first `want`: keys in registers, thread
// i's x-th one number i + x kSelThreads; those past the end are 0 and not counted.
__device__ __forceinline__ uint32_t select_held(const uint32_t (&key)[kSelPer], int cand, int want, int &equal) {
    __shared__ int s_count[2][3][kSelWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t value = 0;  // at least `want` keys are not below it
    int above = 0;       // keys not below value + 2^(shift + 2)
    for (int shift = 30, round = 0; shift >= 0; shift -= 2, round ^= 1) {
        int n[3] = {0, 0, 0};
#pragma unroll
        for (int x = 0; x < kSelPer; ++x) {
            if (x % 8 == 0 && x * kSelThreads >= cand) break;
#pragma unroll
            for (int d = 0; d < 3; ++d) n[d] += key[x] >= value + ((uint32_t)(d + 1) << shift);
        }
#pragma unroll
        for (int d = 0; d < 3; ++d) {
            n[d] = __reduce_add_sync(kFull, n[d]);
            if (lane == 0) s_count[round][d][warp] = n[d];
        }
        __syncthreads();
        int digit = 0;
#pragma unroll
        for (int d = 0; d < 3; ++d) {
            n[d] = __reduce_add_sync(kFull, lane < kSelWarps ? s_count[round][d][lane] : 0);
            if (n[d] >= want) digit = d + 1;
        }
        if (digit < 3) above = n[digit];
        value += (uint32_t)digit << shift;
    }
    equal = want - above;
    return value;
}

// The same by passes over the masses.
__device__ __forceinline__ uint32_t select_read(const KvView &kv, int b, int h, int cand, int want, int &equal) {
    __shared__ int hist[256], s_left;
    __shared__ uint32_t s_value;
    const int tid = threadIdx.x;
    uint32_t value = 0, mask = 0;
    int left = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < cand; i += kSelThreads) {
            const uint32_t k = key_at(kv, b, h, i);
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
    equal = left;
    return value;
}

__global__ void __launch_bounds__(kSelThreads) k_evict_select(const __grid_constant__ EvictArgs a) {
    const KvView &kv = a.kv;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int len = kv.len(b), n = min(len, a.j.budget), fixed = min(a.j.recent, n);
    const int cand = len - fixed, want = n - fixed;
    const int64_t at = (int64_t)b * kv.heads + h;
    int32_t *list = a.list + at * a.j.budget;
    if (h == 0 && tid == 0) a.kept[b] = n;
    for (int i = tid; i < a.chunks; i += kSelThreads) a.loaded[at * a.chunks + i] = 0u;
    if (n == len) {
        for (int i = tid; i < n; i += kSelThreads) list[i] = i;
        return;
    }
    for (int i = tid; i < fixed; i += kSelThreads) list[want + i] = cand + i;
    if (want == 0) return;
    // kept: the keys above value, and the first `equal` equal to it
    __shared__ uint32_t s_warp[kSelPer * kSelWarps];  // of each warp's turn: above, equal << 16
    __shared__ uint2 s_total[kSelWarps];
    if (cand <= kSelPer * kSelThreads) {
        uint32_t key[kSelPer];
#pragma unroll
        for (int x = 0; x < kSelPer; ++x) {
            if (x % 8 == 0 && x * kSelThreads >= cand) break;
            const int i = tid + x * kSelThreads;
            key[x] = i < cand ? key_at(kv, b, h, i) : 0u;
        }
        int equal;
        const uint32_t value = select_held(key, cand, want, equal);
#pragma unroll
        for (int x = 0; x < kSelPer; ++x) {
            if (x % 8 == 0 && x * kSelThreads >= cand) break;
            const bool in = tid + x * kSelThreads < cand;
            const uint32_t gt = __popc(__ballot_sync(kFull, in && key[x] > value));
            const uint32_t eq = __popc(__ballot_sync(kFull, in && key[x] == value));
            if (lane == 0) s_warp[x * kSelWarps + warp] = gt | eq << 16;
        }
        __syncthreads();
        // exclusive scan of all the turns' counts, two a thread
        const int turns = (cand + 8 * kSelThreads - 1) / (8 * kSelThreads) * 8 * kSelWarps;
        uint2 v[2], sum = make_uint2(0u, 0u);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t c = 2 * tid + e < turns ? s_warp[2 * tid + e] : 0u;
            v[e] = make_uint2(c & 0xffffu, c >> 16);
            sum.x += v[e].x;
            sum.y += v[e].y;
        }
        uint2 incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(kFull, incl.x, o), y = __shfl_up_sync(kFull, incl.y, o);
            if (lane >= o) incl.x += x, incl.y += y;
        }
        if (lane == 31) s_total[warp] = incl;
        __syncthreads();
        uint2 pre = make_uint2(incl.x - sum.x, incl.y - sum.y);
        for (int w = 0; w < warp; ++w) pre.x += s_total[w].x, pre.y += s_total[w].y;
        // place of a turn's first key that stays: those above before it, and the equal ones up to their number;
        // and how many of its equal ones stay
        __syncthreads();
        __shared__ int2 s_place[kSelPer * kSelWarps];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            s_place[2 * tid + e] = make_int2((int)pre.x, (int)pre.y);
            pre.x += v[e].x;
            pre.y += v[e].y;
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kSelPer; ++x) {
            if (x % 8 == 0 && x * kSelThreads >= cand) break;
            const int i = tid + x * kSelThreads;
            const bool in = i < cand, above = in && key[x] > value, same = in && key[x] == value;
            const unsigned gt = __ballot_sync(kFull, above), eq = __ballot_sync(kFull, same);
            const int2 p = s_place[x * kSelWarps + warp];
            const int g = p.x + __popc(gt & lanemask_lt()), e = p.y + __popc(eq & lanemask_lt());
            if (above || (same && e < equal)) list[g + min(e, equal)] = i;
        }
        return;
    }
    int equal;
    const uint32_t value = select_read(kv, b, h, cand, want, equal);
    int gt0 = 0, eq0 = 0;
    for (int i0 = 0; i0 < cand; i0 += kSelThreads) {
        const int i = i0 + tid;
        const uint32_t k = i < cand ? key_at(kv, b, h, i) : 0u;
        const unsigned gt = __ballot_sync(kFull, i < cand && k > value), eq = __ballot_sync(kFull, i < cand && k == value);
        if (lane == 0) s_warp[warp] = __popc(gt) | __popc(eq) << 16;
        __syncthreads();
        int g = gt0 + __popc(gt & lanemask_lt()), e = eq0 + __popc(eq & lanemask_lt());
        for (int w = 0; w < kSelWarps; ++w) {
            if (w < warp) g += s_warp[w] & 0xffffu, e += s_warp[w] >> 16;
            gt0 += s_warp[w] & 0xffffu, eq0 += s_warp[w] >> 16;
        }
        if (i < cand && (k > value || (k == value && e < equal))) list[g + min(e, equal)] = i;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const __grid_constant__ EvictArgs a) {
    const KvView &kv = a.kv;
    const int chunk = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int n = a.kept[b], per_part = kv.dim / 8, per = 2 * per_part;
    if (chunk == 0 && h == 0 && tid == 0) a.j.new_lens[b] = n;
    const int r0 = chunk * a.rows, m = min(a.rows, n - r0);
    if (m <= 0) return;
    const int64_t at = (int64_t)b * kv.heads + h;
    const int32_t *list = a.list + at * a.j.budget + r0;
    uint4 x[kMoveChunks];
    char *to[kMoveChunks];
    // of a row, chunks of its key, then of its value
#pragma unroll
    for (int c = 0; c < kMoveChunks; ++c) {
        const int id = tid + c * kMoveThreads, r = id / per, part = id % per;
        to[c] = nullptr;
        if (r >= m) continue;
        const bool v = part >= per_part;
        const int64_t off = (int64_t)(v ? part - per_part : part) * 16;
        const int from = list[r];
        int sp, ss, dp;
        uint32_t q, ds;
        if (!kv.place(b, from, sp, ss)) continue;
        kv.ps.divmod((uint32_t)(r0 + r), q, ds);
        dp = a.j.new_table[b * a.j.new_stride + q];
        if (dp < 0 || dp >= kv.pages) continue;
        if (dp == sp && (int)ds == ss) continue;  // where it is already
        to[c] = (v ? kv.V + dp * kv.v_page + ds * kv.v_slot + h * kv.v_head
                   : kv.K + dp * kv.k_page + ds * kv.k_slot + h * kv.k_head) + off;
        x[c] = *reinterpret_cast<const uint4 *>((v ? kv.V + sp * kv.v_page + ss * kv.v_slot + h * kv.v_head
                                                   : kv.K + sp * kv.k_page + ss * kv.k_slot + h * kv.k_head) + off);
    }
    float w = 0.0f, *wto = nullptr;
    if (tid < m) {
        const int from = list[tid];
        int sp, ss, dp;
        uint32_t q, ds;
        kv.ps.divmod((uint32_t)(r0 + tid), q, ds);
        dp = a.j.new_table[b * a.j.new_stride + q];
        if (kv.place(b, from, sp, ss) && dp >= 0 && dp < kv.pages) {
            w = *kv.mass_at(sp, ss, h);
            wto = kv.mass_at(dp, (int)ds, h);
        }
    }
    uint32_t *loaded = a.loaded + at * a.chunks;
    __threadfence();  // the rows are read before the report
    __syncthreads();
    if (tid == 0) asm volatile("st.release.gpu.global.u32 [%0], 1;" ::"l"(loaded + chunk) : "memory");
    bool ok = true;
    for (int i = tid; i < chunk && ok; i += kMoveThreads) {
        uint32_t spin = 0;
        while (!ld_acquire_u32(loaded + i) && ok) ok = ++spin < kSpinLimit;
    }
    if (!__syncthreads_and(ok)) {
        if (tid == 0) record_error(a.err, kErrScanTimeout);
        return;
    }
#pragma unroll
    for (int c = 0; c < kMoveChunks; ++c)
        if (to[c]) *reinterpret_cast<uint4 *>(to[c]) = x[c];
    if (wto) *wto = w;
}

}  // namespace

cudaError_t launch_evict(const EvictJob &j, const KvView &kv, cudaStream_t s) {
    EvictArgs a{};
    a.j = j;
    a.kv = kv;
    a.err = library_error_word();
    if (!a.err) return cudaErrorUnknown;
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d;
    if (a.j.budget > room) a.j.budget = (int)room;  // no sequence is longer
    // rows of a CTA: whole ones, no more than it has threads for their masses
    a.rows = kMoveThreads * kMoveChunks / (kv.dim / 4);
    if (a.rows > kMoveThreads) a.rows = kMoveThreads;
    a.chunks = (a.j.budget + a.rows - 1) / a.rows;
    void *p = nullptr;
    const size_t lists = (size_t)kv.B * kv.heads * a.j.budget;
    const size_t flags = (size_t)kv.B * kv.heads * a.chunks;
    const cudaError_t e = stream_scratch(kScratchAttention, (lists + kv.B + flags) * sizeof(int32_t), s, &p);
    if (e != cudaSuccess) return e;
    a.list = static_cast<int32_t *>(p);
    a.kept = a.list + lists;
    a.loaded = reinterpret_cast<uint32_t *>(a.kept + kv.B);
    k_evict_select<<<dim3((unsigned)kv.heads, (unsigned)kv.B), kSelThreads, 0, s>>>(a);
    const cudaError_t e1 = counted_launch(cudaGetLastError());
    if (e1 != cudaSuccess) return e1;
    return launch_dependent(k_evict_move, dim3((unsigned)a.chunks, (unsigned)kv.heads, (unsigned)kv.B), kMoveThreads, a, s);
}

}  // namespace pv
