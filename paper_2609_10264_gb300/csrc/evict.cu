// Eviction from a paged cache by accumulated attention weight (pvmvmd_kv_evict).
//
// k_evict_select, a CTA per (sequence, head): the kept tokens' indexes, ascending.
// Masses map to integers of the same order, held in registers (up to 32768 of them;
// those of longer sequences are read again for every pass).  The value of the last
// one kept is found in three passes of 11, 11 and 10 bits: a histogram of the keys
// that share the digits found, and a scan of its bins.  Another scan over the counts
// of every warp's keys gives each kept one its place.
//
// k_evict_move: the rows of a list, 16 KiB of keys and as many of values a CTA.  A row
// never moves to a higher index, so in place the rows that lie where a CTA writes are
// its own or those of CTAs before it: every CTA reports its rows read, and one that
// writes to a page that the sequence has in that very place waits for the reports
// before its own first.
// Blocks start in the order of their index (as the other kernels that chain blocks
// rest on); the wait is bounded.  16 sequences of up to 16384 keys to 4096: 110 us a call to
// other pages, 4.6 TB/s of rows read and written, and 152 in place, of which the waits for
// the CTAs before are the difference; one of 700 keys 9.4 us, latency of both kernels.
// To a quarter: 8 sequences of 32768 masses, in registers, 140 us, of 33024, read again,
// 140; one of 131072 389.
#include <algorithm>

#include "attention.cuh"

namespace pv {
namespace {

constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32;
constexpr int kSelPer = 32;   // keys per thread in registers
constexpr int kBins = 2048;
constexpr int kMoveThreads = 128;
constexpr int kMoveBytes = 32 << 10;  // of keys and values per CTA

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

// Sum of v over the threads before this one, and over all.
template <typename V>
__device__ __forceinline__ V scan_before(V v, V &total) {
    __shared__ V s_warp[kSelWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V x = __shfl_up_sync(kFull, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    V w = s_warp[lane];
    static_assert(kSelWarps == 32, "a lane per warp");
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V x = __shfl_up_sync(kFull, w, o);
        if (lane >= o) w += x;
    }
    total = __shfl_sync(kFull, w, 31);
    const V before = __shfl_sync(kFull, w, warp ? warp - 1 : 0);
    __syncthreads();
    return (warp ? before : V(0)) + incl - v;
}

// A key into its bin; by whole warps.  Lanes of one bin (equal masses) add once.
__device__ __forceinline__ void count_key(int *hist, bool in, int bin) {
    int same;
    __match_all_sync(kFull, in ? bin : -1, &same);
    if (in && (!same || (threadIdx.x & 31) == 0)) atomicAdd(&hist[bin], same ? 32 : 1);
}

// The largest value of which at least `want` of the keys are not below, and how many
// of those equal to it are among them: those that `each` shows, want at least one.
template <typename Each>
__device__ __forceinline__ uint32_t select(Each each, int want, int &equal) {
    __shared__ int hist[kBins];
    __shared__ uint32_t s_value;
    __shared__ int s_left;
    const int tid = threadIdx.x;
    uint32_t value = 0, mask = 0;
    int left = want;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        const uint32_t bits = pass == 2 ? 0x3ffu : kBins - 1u;
        each([&](bool in, uint32_t key) { count_key(hist, in && (key & mask) == value, (int)((key >> shift) & bits)); });
        __syncthreads();
        // bins from the top
        const int b0 = kBins - 1 - 2 * tid;
        const int c0 = hist[b0], c1 = hist[b0 - 1];
        int total;
        const int above = scan_before(c0 + c1, total);
        if (above < left && left <= above + c0 + c1) {
            const bool second = left > above + c0;
            s_value = value | (uint32_t)(second ? b0 - 1 : b0) << shift;
            s_left = left - above - (second ? c0 : 0);
        }
        __syncthreads();
        value = s_value;
        left = s_left;
        mask |= bits << shift;
    }
    equal = left;
    return value;
}

__global__ void __launch_bounds__(kSelThreads) k_evict_select(const __grid_constant__ EvictArgs a) {
    const KvView &kv = a.kv;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    follow();
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
    if (cand <= kSelPer * kSelThreads) {
        __shared__ uint32_t s_turn[kSelPer * kSelWarps];  // of a warp's turn: above, equal << 16; then their places
        __shared__ int2 s_place[kSelPer * kSelWarps];
        uint32_t key[kSelPer];
        const int turns = (cand + kSelThreads - 1) / kSelThreads;
#pragma unroll
        for (int x = 0; x < kSelPer; x += 4) {
            if (x >= turns) break;
            int page[4], slot[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {  // (one past the end looks where the last one does)
                const int i = min(tid + (x + y) * kSelThreads, cand - 1);
                if (!kv.place(b, i, page[y], slot[y])) page[y] = -1;
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const float v = *kv.mass_at(max(page[y], 0), slot[y], h);
                key[x + y] = page[y] >= 0 ? mass_key(v) : 0u;
            }
        }
        int equal;
        const uint32_t value = select(
            [&](auto count) {
#pragma unroll
                for (int x = 0; x < kSelPer; ++x) {
                    if (x >= turns) break;
                    count(tid + x * kSelThreads < cand, key[x]);
                }
            },
            want, equal);
#pragma unroll
        for (int x = 0; x < kSelPer; ++x) {
            if (x >= turns) break;
            const bool in = tid + x * kSelThreads < cand;
            const uint32_t gt = __popc(__ballot_sync(kFull, in && key[x] > value));
            const uint32_t eq = __popc(__ballot_sync(kFull, in && key[x] == value));
            if (lane == 0) s_turn[x * kSelWarps + warp] = gt | eq << 16;
        }
        __syncthreads();
        const uint32_t c = tid < turns * kSelWarps ? s_turn[tid] : 0u;
        unsigned long long total;
        const unsigned long long pre =
            scan_before((unsigned long long)(c & 0xffffu) | (unsigned long long)(c >> 16) << 32, total);
        s_place[tid] = make_int2((int)(uint32_t)pre, (int)(pre >> 32));
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kSelPer; ++x) {
            if (x >= turns) break;
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
    const uint32_t value = select(
        [&](auto count) {
            for (int i0 = 0; i0 < cand; i0 += kSelThreads) count(i0 + tid < cand, i0 + tid < cand ? key_at(kv, b, h, i0 + tid) : 0u);
        },
        want, equal);
    int gt0 = 0, eq0 = 0;
    for (int i0 = 0; i0 < cand; i0 += kSelThreads) {
        const int i = i0 + tid;
        const uint32_t k = i < cand ? key_at(kv, b, h, i) : 0u;
        const bool above = i < cand && k > value, same = i < cand && k == value;
        unsigned long long total;
        const unsigned long long pre =
            scan_before((unsigned long long)above | (unsigned long long)same << 32, total);
        const int g = gt0 + (int)(uint32_t)pre, e = eq0 + (int)(pre >> 32);
        if (above || (same && e < equal)) list[g + min(e, equal)] = i;
        gt0 += (int)(uint32_t)total;
        eq0 += (int)(total >> 32);
    }
}

__global__ void __launch_bounds__(kMoveThreads) k_evict_move(const __grid_constant__ EvictArgs a) {
    const KvView &kv = a.kv;
    const int chunk = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    extern __shared__ __align__(16) uint8_t smem[];
    // where each row is and goes
    __shared__ int64_t s_from[2][kMoveThreads], s_to[2][kMoveThreads];
    const int r0 = chunk * a.rows, per_part = kv.dim / 8, per = 2 * per_part;  // 16-byte chunks
    static_assert(2 * PVMVMD_MAX_HEAD / 8 <= 32, "a lane per chunk");
    const int64_t at = (int64_t)b * kv.heads + h;
    uint32_t q, o;
    kv.ps.divmod((uint32_t)(r0 + tid), q, o);
    const int ds = (int)o;
    follow();
    const int n = a.kept[b];
    const int from = tid < a.rows && r0 + tid < a.j.budget ? a.list[at * a.j.budget + r0 + tid] : 0;
    if (chunk == 0 && h == 0 && tid == 0) a.j.new_lens[b] = n;
    const int m = min(a.rows, n - r0);
    if (m <= 0) return;
    float w = 0.0f, *wto = nullptr;
    bool own = false;  // goes to a page of the sequence
    if (tid < m) {
        const int dp = a.j.new_table[b * a.j.new_stride + q];
        int sp = 0, ss = 0;
        own = dp == kv.table[b * kv.table_stride + q];
        const bool moves = kv.place(b, from, sp, ss) && dp >= 0 && dp < kv.pages && (dp != sp || ds != ss);
        if (moves) {
            w = *kv.mass_at(sp, ss, h);
            wto = kv.mass_at(dp, ds, h);
        }
        s_from[0][tid] = moves ? sp * kv.k_page + ss * kv.k_slot : -1;
        s_from[1][tid] = sp * kv.v_page + ss * kv.v_slot;
        s_to[0][tid] = dp * kv.k_page + ds * kv.k_slot;
        s_to[1][tid] = dp * kv.v_page + ds * kv.v_slot;
    }
    own = __syncthreads_or(own);
    // a row a warp: the chunks of its key, then of its value, a lane each
    const int lane = tid & 31, warp = tid >> 5;
    const bool v = lane >= per_part;
    char *pool = (v ? kv.V + h * kv.v_head : kv.K + h * kv.k_head) + (v ? lane - per_part : lane) * 16;
    const uint32_t mine = smem_addr(smem) + 16 * lane;
#pragma unroll 4
    for (int r = warp; r < m; r += kMoveThreads / 32)
        if (s_from[0][r] != -1 && lane < per) copy16(mine + 16 * per * r, pool + s_from[v][r], true);
    copy_commit();
    copy_wait<0>();
    uint32_t *loaded = a.loaded + at * a.chunks;
    __threadfence();  // the rows are read before the report
    __syncthreads();
    if (tid == 0) asm volatile("st.release.gpu.global.u32 [%0], 1;" ::"l"(loaded + chunk) : "memory");
    bool ok = true;
    for (int i = tid; own && i < chunk && ok; i += kMoveThreads) {
        uint32_t spin = 0;
        while (!ld_acquire_u32(loaded + i) && ok) ok = ++spin < kSpinLimit;
    }
    if (!__syncthreads_and(ok)) {
        if (tid == 0) record_error(a.err, kErrScanTimeout);
        return;
    }
#pragma unroll 4
    for (int r = warp; r < m; r += kMoveThreads / 32)
        if (s_from[0][r] != -1 && lane < per)
            *reinterpret_cast<uint4 *>(pool + s_to[v][r]) = *reinterpret_cast<const uint4 *>(smem + 16 * (per * r + lane));
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
    a.rows = std::min(kMoveBytes / (4 * kv.dim), kMoveThreads);
    a.chunks = (a.j.budget + a.rows - 1) / a.rows;
    void *p = nullptr;
    const size_t lists = (size_t)kv.B * kv.heads * a.j.budget;
    const size_t flags = (size_t)kv.B * kv.heads * a.chunks;
    const cudaError_t e = stream_scratch(kScratchAttention, (lists + kv.B + flags) * sizeof(int32_t), s, &p);
    if (e != cudaSuccess) return e;
    a.list = static_cast<int32_t *>(p);
    a.kept = a.list + lists;
    a.loaded = reinterpret_cast<uint32_t *>(a.kept + kv.B);
    const cudaError_t e1 =
        launch_dependent(k_evict_select, dim3((unsigned)kv.heads, (unsigned)kv.B), kSelThreads, 0, s, a);
    if (e1 != cudaSuccess) return e1;
    return launch_dependent(k_evict_move, dim3((unsigned)a.chunks, (unsigned)kv.heads, (unsigned)kv.B), kMoveThreads,
                            kMoveBytes, s, a);
}

}  // namespace pv
