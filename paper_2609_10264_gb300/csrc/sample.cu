// The choice of the next token (pvmvmd_sample).
//
// A cluster of CTAs takes a row.  Weights are whole numbers, so their sums are the same in any
// order, and no result depends on the order of atomic operations or of a list.
//
// Without top-k and top-p a row is read twice: for the largest x, and for the weights' sum; then the warp's
// share where the choice falls is read once more.  Bound by the arithmetic of the weights.
// With them, the threads' largest values, four a thread, say where about the k-th largest lies (there are at least k
// values above the k-th largest of them); the second reading puts the tokens up to there into a list, of a few
// times k, and the first CTA finds limits and choice in it: by histograms, whose one bin
// that a limit falls into is resolved by comparing its members with one another.
// Where the list does not hold what the limits leave (flat rows, a large k), the limit is looked
// for digit by digit in all values, each digit another reading.
#include "rows.cuh"

namespace pv {
namespace {

constexpr int kSThreads = 512, kSWarps = kSThreads / 32;
constexpr int kBins = 2048;
constexpr int kList = 4096;      // tokens of the list
constexpr int kMostK = 1024;     // a larger k (twice of it with several CTAs) is not looked for in a list
constexpr int kMembers = 1024;   // of a bin at most that are compared with one another
constexpr int kTopPList = 768;   // tokens that are put in a list for top-p alone, about
constexpr int kGroups = 4;       // largest values that a thread keeps
using u64 = unsigned long long;

struct SampleShared {
    u64 bins[kBins];
    uint32_t counts[kBins];
    float x[kList], bin_x[kList];    // the list; one bin's members
    int index[kList], bin_index[kList];
    u64 warp[kSWarps], cta, before, weight, kept;
    uint32_t warp_count[kSWarps], found, key[kSWarps], ctakey, count, members, cut_index, general;
    float cut_x;
};

__device__ __forceinline__ u64 peer_u64(const u64 *p, uint32_t rank) {
    uint32_t a;
    u64 v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t peer_u32(const uint32_t *p, uint32_t rank) {
    uint32_t a, v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// 32-bit numbers in order, as whole numbers; NaN is not among them.  (Adding 0 makes the two zeros one.)
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.0f));
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
    return __uint_as_float(k ^ (k & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
constexpr uint32_t kNoKey = 0x007fffffu;  // of -infinity

// W of a token: 2^-(big - x) in units of 2^-40.
__device__ __forceinline__ u64 weight(float big, float x) {
    Two sum;
    const Two f = split(both(fminf(__fsub_rn(big, x), 63.0f)), sum);
    const float r = __fadd_rn(first(exp_poly(f, 4194304.0f)), 8388608.0f);  // 2^23 + round(2^22 P)
    return ((u64)(__float_as_uint(r) & 0x7fffffu) << 18) >> ((uint32_t)sum.v - 0x4b400000u);
}
__device__ __forceinline__ uint32_t shift_left(uint32_t v, uint32_t n) {  // 0 from 32 on
    uint32_t r;
    asm("shl.b32 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(n));
    return r;
}
__device__ __forceinline__ uint32_t shift_right(uint32_t v, uint32_t n) {
    uint32_t r;
    asm("shr.u32 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(n));
    return r;
}
// floor(v f / 2^31), f < 2^31
__device__ __forceinline__ u64 part_of(u64 v, uint32_t f31) { return __umul64hi(v, (u64)f31 << 33); }
// floor(2^31 p) of a part in [0, 1]
__device__ __forceinline__ uint32_t part31(float p) {
    return p > 0.0f ? (uint32_t)__fmul_rn(fminf(p, 1.0f), 2147483648.0f) : 0u;
}
// The bin of a distance d >= 0: 2^kFine of them between one power of two and the next, from 2^-10 to 2^6; what is below is in
// the first one.
template <int kFine>
__device__ __forceinline__ int bin_of(float d) {
    const int b = (int)(__float_as_uint(d) >> (23 - kFine)) - (117 << kFine);
    return min(max(b, 0), (16 << kFine) - 1);
}
// d is in a bin up to b exactly where d < this.
template <int kFine>
__device__ __forceinline__ float bin_end(int b) {
    return __uint_as_float((uint32_t)(b + 1 + (117 << kFine)) << (23 - kFine));
}

struct SampleArgs {
    SampleJob j;
    int ctas;  // of a row
};

template <int kType>
struct Row;
template <int kType>
__device__ __noinline__ void limits_by_digits(Row<kType> r, int top_k, float top_p, u64 least);

// kType: the logits', all of which are allowed and have no scales of their own; or kAny, and anything.
template <int kType>
struct Row {
    const SampleArgs &a;
    SampleShared &sh;
    int64_t t;
    int lane, warp, type;
    uint32_t rank, ctas;
    const char *base;  // the 16-byte boundary at or before the row
    int off, end;      // the row's tokens are off .. end - 1 from there
    int begin, last;   // tiles of this warp
    float m;
    const uint32_t *allowed;
    float big;         // the largest x
    uint32_t top;      // its key

    __device__ __forceinline__ void meet() const {
        if (ctas > 1)
            clusters_meet();
        else
            __syncthreads();
    }
    // This warp's tiles that lie in the row whole: from .. to - 1 (from <= to).
    __device__ __forceinline__ int whole_from() const { return min(last, max(begin, (off + kTile - 1) / kTile)); }
    __device__ __forceinline__ int whole_to() const { return max(whole_from(), min(last, end / kTile)); }
    __device__ __forceinline__ Raw load_inside(int tile) const {
        Raw r;
        const char *p = base + (int64_t)(tile * kTile + lane * kWide) * (two_bytes(type) ? 2 : 4);
        r.a = *reinterpret_cast<const uint4 *>(p);
        if (!two_bytes(type)) r.b = *reinterpret_cast<const uint4 *>(p + 16);
        return r;
    }
    // x of a lane's eight tokens of a tile, -infinity where there is none or it may not be chosen;
    // the first one's index.
    __device__ __forceinline__ int tokens(int tile, float (&x)[kWide]) const {
        const pvmvmd_rows &l = a.j.logits;
        const int at = tile * kTile + lane * kWide;
        Raw r;
        r.a = r.b = make_uint4(0, 0, 0, 0);
        if (two_bytes(type)) {
            if (at < end && at + kWide > off) r.a = *reinterpret_cast<const uint4 *>(base + (int64_t)at * 2);
        } else {
            if (at < end && at + 4 > off) r.a = *reinterpret_cast<const uint4 *>(base + (int64_t)at * 4);
            if (at + 4 < end && at + 8 > off) r.b = *reinterpret_cast<const uint4 *>(base + (int64_t)at * 4 + 16);
        }
        Two v2[kTwos];
        unpack(r, type, v2);
        const int i0 = at - off, V = a.j.V;
        uint32_t ok = 0xff;
        if (kType == kAny && allowed) {
            const int w = i0 >> 5, words = (V + 31) >> 5;
            const uint32_t lo = w >= 0 && w < words ? allowed[w] : 0u;
            const uint32_t hi = (i0 & 31) > 24 && w + 1 < words ? allowed[w + 1] : 0u;
            ok = __funnelshift_r(lo, hi, i0 & 31);
        }
#pragma unroll
        for (int e = 0; e < kWide; ++e) {
            float v = __fmul_rn(e & 1 ? second(v2[e / 2]) : first(v2[e / 2]), m);
            const bool in = i0 + e >= 0 && i0 + e < V;
            if (kType == kAny && l.channel_scale_dev && in) v = __fmul_rn(v, l.channel_scale_dev[i0 + e]);
            v = v > -INFINITY ? fminf(v, kFltMax) : -INFINITY;  // (NaN is not)
            x[e] = in && (ok >> e & 1) ? v : -INFINITY;
        }
        return i0;
    }
    // The same for a tile inside the row and kType, from what load_inside gave, without the cut at FLT_MAX: NaN and
    // infinities as they come.
    __device__ __forceinline__ void plain_tokens(const Raw &r, Two (&x)[kTwos]) const {
        unpack(r, type, x);
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = mul2(x[i], both(m));
    }

    // f(x, index) for every token of this warp's tiles that may be chosen
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
        for (int k = begin; k < last; ++k) {
            float x[kWide];
            const int i0 = tokens(k, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e)
                if (x[e] > -INFINITY) f(x[e], i0 + e);
        }
    }

    __device__ __forceinline__ uint32_t max_key(uint32_t k) const {
        k = __reduce_max_sync(kFull, k);
        if (lane == 0) sh.key[warp] = k;
        __syncthreads();
        k = __reduce_max_sync(kFull, lane < kSWarps ? sh.key[lane] : 0u);
        if (ctas > 1) {
            if (threadIdx.x == 0) sh.ctakey = k;
            clusters_meet();
            k = __reduce_max_sync(kFull, lane < (int)ctas ? peer_u32(&sh.ctakey, (uint32_t)lane) : 0u);
        }
        meet();
        return k;
    }

    // The largest x of a thread's tokens in kGroups parts of them (-infinity: none).
    __device__ __forceinline__ void largest(float (&g)[kGroups]) const {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) g[i] = -INFINITY;
        int k = begin;
        auto edge = [&](int tile) {
            float x[kWide];
            tokens(tile, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e) g[e % kGroups] = fmaxf(g[e % kGroups], x[e]);
        };
        if (kType != kAny && m > 0.0f) {
            // rounding keeps the order, so that the largest logit has the largest x
            const int from = whole_from(), to = whole_to();
            for (; k < from; ++k) edge(k);
            if (from < to) {
                uint32_t n[kGroups];
                float v[kGroups];
                auto take = [&](const Raw &r, bool start) {
                    const uint32_t w[kWide] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
                    for (int i = 0; i < kGroups; ++i) {
                        if (kType == kBf16) {
                            const __nv_bfloat162 p = *reinterpret_cast<const __nv_bfloat162 *>(&w[i]);
                            const __nv_bfloat162 q = start ? p : __hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&n[i]), p);
                            n[i] = *reinterpret_cast<const uint32_t *>(&q);
                        } else if (kType == kF16) {
                            const __half2 p = *reinterpret_cast<const __half2 *>(&w[i]);
                            const __half2 q = start ? p : __hmax2(*reinterpret_cast<const __half2 *>(&n[i]), p);
                            n[i] = *reinterpret_cast<const uint32_t *>(&q);
                        } else if (kType == kF32) {
                            const float p = fmaxf(__uint_as_float(w[i]), __uint_as_float(w[i + 4]));
                            v[i] = start ? p : fmaxf(v[i], p);
                        } else {  // less the smallest, field elements are in the order of their integers
                            const uint32_t p = max(w[i] - (kHalfQ + 1), w[i + 4] - (kHalfQ + 1));
                            n[i] = start ? p : max(n[i], p);
                        }
                    }
                };
                take(load_inside(k++), true);
#pragma unroll 4
                for (; k < to; ++k) take(load_inside(k), false);
#pragma unroll
                for (int i = 0; i < kGroups; ++i) {
                    float p;
                    if (kType == kBf16 || kType == kF16) {
                        const Two h = kType == kBf16 ? bfloat2_of(n[i]) : half2_of(n[i]);
                        p = fmaxf(first(h), second(h));
                    } else {
                        p = kType == kF32 ? v[i] : to_f32<uint32_t>(n[i] + (kHalfQ + 1));
                    }
                    p = __fmul_rn(p, m);
                    if (p > -INFINITY) g[i] = fmaxf(g[i], fminf(p, kFltMax));  // (a part of NaN alone stays as it was)
                }
            }
        }
#pragma unroll 1
        for (; k < last; ++k) edge(k);
    }

    // One pass over the warp's tiles: sum, where asked for, of the weights that are at least `least`; and collect(x,
    // index) for the tokens nearer than `near`.
    template <bool kSum, bool kCollect, typename C>
    __device__ __forceinline__ u64 pass(u64 least, float near, C collect) const {
        u64 sum = 0;
        int k = begin;
        auto edge = [&](int tile) {
            float x[kWide];
            const int i0 = tokens(tile, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e) {
                if (x[e] > -INFINITY) {
                    if (kSum) {
                        const u64 w = weight(big, x[e]);
                        sum += w >= least ? w : 0ull;
                    }
                    if (kCollect && __fsub_rn(big, x[e]) < near) collect(x[e], i0 + e);
                }
            }
        };
        if (kType != kAny && big < kFltMax) {  // (no x is cut)
            const int from = whole_from(), to = whole_to();
            for (; k < from; ++k) edge(k);
#pragma unroll 2
            for (; k < to; ++k) {
                Two x[kTwos];
                plain_tokens(load_inside(k), x);
                uint32_t hits = 0, low = 0;
#pragma unroll
                for (int i = 0; i < kTwos; ++i) {
                    Two d = sub2(both(big), x[i]);
                    if (kCollect) hits |= (first(d) < near ? 1u << 2 * i : 0u) | (second(d) < near ? 2u << 2 * i : 0u);
                    if (kSum) {
                        d = two(fminf(first(d), 63.0f), fminf(second(d), 63.0f));  // (NaN: 63)
                        Two n;
                        const Two r = add2(exp_poly(split(d, n), 4194304.0f), both(8388608.0f));
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t p = (uint32_t)(h ? r.v >> 32 : r.v) & 0x7fffffu, q = (uint32_t)(h ? n.v >> 32 : n.v);
                            if (least) {
                                const u64 w = ((u64)p << 18) >> (q - 0x4b400000u);
                                sum += w >= least ? w : 0ull;
                            } else {  // p 2^(18 - n) for n < 18; the others are below 2^23
                                sum += (u64)p * shift_left(2u, 0x4b400000u + 17u - q);
                                low += shift_right(p, q - (0x4b400000u + 18u));
                            }
                        }
                    }
                }
                if (kSum) sum += low;
                if (kCollect && hits) {
                    const int i0 = k * kTile + lane * kWide - off;
#pragma unroll
                    for (int e = 0; e < kWide; ++e)
                        if (hits >> e & 1) collect(e & 1 ? second(x[e / 2]) : first(x[e / 2]), i0 + e);
                }
            }
        }
#pragma unroll 1
        for (; k < last; ++k) edge(k);
        return sum;
    }

    // Bins' sums from the front: of a thread's four (of 2048).  pre: in front of the first of them.
    template <typename T>
    __device__ __forceinline__ T scan(const T (&mine)[kBins / kSThreads], T *warps, T &total) const {
        T sum = 0;
#pragma unroll
        for (int i = 0; i < kBins / kSThreads; ++i) sum += mine[i];
        T pre = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T u = __shfl_up_sync(kFull, pre, o);
            if (lane >= o) pre += u;
        }
        if (lane == 31) warps[warp] = pre;
        __syncthreads();
        pre -= sum;
        total = 0;
#pragma unroll
        for (int k = 0; k < kSWarps; ++k) {
            const T w = warps[k];
            if (k < warp) pre += w;
            total += w;
        }
        return pre;
    }

    // The smallest value v up to which `target` is reached by the weights of all tokens with values up
    // to v; what those below v and at v weigh.  f(x, index, value, weight) says whether a token takes part.  False
    // where all together do not reach it (before: what they weigh).
    template <typename F>
    __device__ __forceinline__ bool reach(int bits, u64 target, F f, uint32_t &v, u64 &before, u64 &at) const {
        v = 0;
        before = at = 0;
        uint32_t open = 0;  // bits not looked at yet
        for (int left = bits; left > 0; left = (int)open) {
            const int digit = min(left, 11);
            open = (uint32_t)(left - digit);
            for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.bins[i] = 0;
            if (threadIdx.x == 0) sh.found = ~0u;
            __syncthreads();
            const uint32_t high = v;
            each([&](float x, int i) {
                uint32_t value;
                u64 w;
                if (f(x, i, value, w) && ((u64)value >> left) == ((u64)high >> left) && w)
                    atomicAdd(&sh.bins[(value >> open) & ((1u << digit) - 1)], w);
            });
            meet();
            constexpr int kMine = kBins / kSThreads;
            u64 mine[kMine], total;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int b = (int)threadIdx.x * kMine + i;
                mine[i] = 0;
                for (uint32_t c = 0; c < ctas; ++c) mine[i] += ctas > 1 ? peer_u64(&sh.bins[b], c) : sh.bins[b];
            }
            u64 pre = before + scan(mine, sh.warp, total);
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                if (pre < target && pre + mine[i] >= target) {
                    sh.found = threadIdx.x * kMine + i;
                    sh.before = pre;
                    sh.weight = mine[i];
                }
                pre += mine[i];
            }
            meet();  // (the bins have been read, too)
            if (sh.found == ~0u) {  // in the first digit alone
                before += total;
                __syncthreads();
                return false;
            }
            v |= sh.found << open;
            before = sh.before;
            at = sh.weight;
            __syncthreads();
        }
        return true;
    }

    // One token, its weight and that of all that are kept: the row's results, by the thread that has them.
    __device__ __forceinline__ void choose(int index, u64 w, u64 Z) const {
        a.j.token[t] = index;
        if (a.j.logprob) a.j.logprob[t] = -log1pf(__fdiv_rn((float)(Z - w), (float)w));
    }
    __device__ __forceinline__ u64 random_part(u64 Z) const { return __umul64hi(Z, (u64)a.j.random[t] << 32); }

    // The choice among the tokens that kept(x, index) gives a weight to, `sum` being that of this warp's.
    template <typename F>
    __device__ __forceinline__ void choose_in_order(u64 sum, F kept) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        __syncthreads();
        if (lane == 0) sh.warp[warp] = sum;
        __syncthreads();
        u64 mine = 0, front = 0, Z = 0;  // of this CTA; of the CTAs in front; of all
#pragma unroll
        for (int k = 0; k < kSWarps; ++k) mine += sh.warp[k];
        if (ctas > 1) {
            if (threadIdx.x == 0) sh.cta = mine;
            clusters_meet();
            for (uint32_t c = 0; c < ctas; ++c) {
                const u64 v = peer_u64(&sh.cta, c);
                if (c < rank) front += v;
                Z += v;
            }
            clusters_meet();  // nothing of a CTA's is read once it may have ended
        } else {
            Z = mine;
        }
        const u64 at = random_part(Z);
        if (at < front || at >= front + mine) return;  // another CTA's
        // the warp whose tiles they are, and then all warps on parts of these
        int owner = 0;
#pragma unroll
        for (int k = 0; k < kSWarps - 1; ++k) {
            const u64 w = sh.warp[k];
            if (owner == k && at >= front + w) {
                front += w;
                owner = k + 1;
            }
        }
        const int per = (last_of(owner) - begin_of(owner) + kSWarps - 1) / kSWarps;
        const int from = min(last_of(owner), begin_of(owner) + warp * per), to = min(last_of(owner), from + per);
        auto weights = [&](int k, u64 (&w)[kWide]) {
            float x[kWide];
            const int i0 = tokens(k, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e) w[e] = x[e] > -INFINITY ? kept(x[e], i0 + e) : 0ull;
            return i0;
        };
        u64 part = 0;
#pragma unroll 1
        for (int k = from; k < to; ++k) {
            u64 w[kWide];
            weights(k, w);
#pragma unroll
            for (int e = 0; e < kWide; ++e) part += w[e];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(kFull, part, o);
        __syncthreads();
        if (lane == 0) sh.warp[warp] = part;
        __syncthreads();
        for (int k = 0; k < warp; ++k) front += sh.warp[k];
        if (at < front || at >= front + part) return;
#pragma unroll 1
        for (int k = from; k < to; ++k) {
            u64 w[kWide], all = 0;
            const int i0 = weights(k, w);
#pragma unroll
            for (int e = 0; e < kWide; ++e) all += w[e];
            u64 pre = all;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 u = __shfl_up_sync(kFull, pre, o);
                if (lane >= o) pre += u;
            }
            const u64 tile = __shfl_sync(kFull, pre, 31);
            pre += front - all;
            if (at >= pre && at < pre + all) {
#pragma unroll
                for (int e = 0; e < kWide; ++e) {
                    if (at >= pre && at < pre + w[e]) choose(i0 + e, w[e], Z);
                    pre += w[e];
                }
            }
            front += tile;
            if (at < front) return;
        }
    }
    int tiles, share;  // the row's, and a warp's
    __device__ __forceinline__ int begin_of(int w) const { return min(tiles, ((int)rank * kSWarps + w) * share); }
    __device__ __forceinline__ int last_of(int w) const { return min(tiles, begin_of(w) + share); }

    // The limits looked for in all values.
    __device__ __forceinline__ void general(int top_k, float top_p, u64 least) {
        // What is kept: values below cut, and of those at it the tokens up to cut_index.
        uint32_t cut = ~0u, cut_index = ~0u;
        u64 ties = 0, at_cut = 0;  // how many of those at it are kept; how many there are
        u64 before, at;
        if (top_k && reach(32, (u64)top_k, [&](float x, int, uint32_t &v, u64 &w) {
                v = top - key_of(x);
                w = 1;
                return true;
            }, cut, before, at)) {
            ties = (u64)top_k - before;
            at_cut = at;
        } else {
            cut = ~0u;
        }
        if (top_p < 1.0f) {
            auto below = [&](float x, int, uint32_t &v, u64 &w) {
                v = top - key_of(x);
                w = weight(big, x);
                return v < cut;
            };
            // (what is below the cut, from a target that is not reached)
            uint32_t v;
            reach(32, ~0ull, below, v, before, at);
            const u64 each = weight(big, of_key(top - cut)), kept = before + (cut == ~0u ? 0 : ties * each);
            const u64 target = max(part_of(kept, part31(top_p)), 1ull);
            if (reach(32, target, below, v, before, at)) {
                const u64 one = weight(big, of_key(top - v));
                cut = v;
                at_cut = at / one;
                ties = (target - before + one - 1) / one;
            } else {
                ties = (target - before + each - 1) / each;  // among those that top-k leaves at its cut
            }
        }
        if (cut != ~0u && ties < at_cut) {
            u64 b, w1;
            uint32_t index;
            reach(24, ties, [&](float x, int i, uint32_t &v, u64 &w) {
                v = (uint32_t)i;
                w = 1;
                return top - key_of(x) == cut;
            }, index, b, w1);
            cut_index = index;
        }
        auto kept = [&](float x, int i) {
            const uint32_t v = top - key_of(x);
            const u64 w = weight(big, x);
            return (v < cut || (v == cut && (uint32_t)i <= cut_index)) && w >= least ? w : 0ull;
        };
        u64 sum = 0;
        each([&](float x, int i) { sum += kept(x, i); });
        choose_in_order(sum, kept);
    }

    // ------------------------------------------------------------ the list
    // The list's tokens of thread threadIdx.x: f(x, index).
    template <typename F>
    __device__ __forceinline__ void listed(int n, F f) const {
        for (int i = threadIdx.x; i < n; i += kSThreads) f(sh.x[i], sh.index[i]);
    }
    // Those that in(x, index) takes, to bin_x and bin_index.  (A barrier in front of it and after it.)
    template <typename F>
    __device__ __forceinline__ int gather(int n, F in) const {
        if (threadIdx.x == 0) sh.members = 0;
        __syncthreads();
        listed(n, [&](float x, int i) {
            if (in(x, i)) {
                const uint32_t p = atomicAdd(&sh.members, 1u);
                sh.bin_x[p] = x;
                sh.bin_index[p] = i;
            }
        });
        __syncthreads();
        return (int)sh.members;
    }
    static __device__ __forceinline__ bool ahead(float x, int i, float y, int k) { return x > y || (x == y && i < k); }

    // The choice from a list of n tokens, which are all those nearer than the first one that is not there.  total: what
    // all tokens of the row weigh, 0 where top_k limits them.  False where the limits leave more than the list, or
    // too many fall into one bin.
    __device__ __forceinline__ bool choose_listed(int n, int top_k, float top_p, u64 least, u64 total) {
        constexpr int kMine = kBins / kSThreads;
        for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.bins[i] = 0, sh.counts[i] = 0;
        if (threadIdx.x == 0) {
            sh.found = ~0u;
            sh.cut_x = -INFINITY;
            sh.cut_index = ~0u;
            sh.kept = 0;
        }
        __syncthreads();
        listed(n, [&](float x, int) {
            const int b = bin_of<7>(__fsub_rn(big, x));
            atomicAdd(&sh.bins[b], weight(big, x));
            atomicAdd(&sh.counts[b], 1u);
        });
        __syncthreads();
        u64 mass[kMine], all;
        uint32_t count[kMine], number;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            mass[i] = sh.bins[threadIdx.x * kMine + i];
            count[i] = sh.counts[threadIdx.x * kMine + i];
        }
        const uint32_t pre_count = scan(count, sh.warp_count, number);
        const u64 pre_mass = scan(mass, sh.warp, all);
        u64 S = total ? total : all;  // what top-k leaves
        u64 in_front = ~0ull;         // of top-k's bin
        int k_bin = kBins, members = 0, keep = 0;
        if (top_k && (uint32_t)top_k < number) {
            uint32_t c = pre_count;
            u64 w = pre_mass;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                if (c < (uint32_t)top_k && c + count[i] >= (uint32_t)top_k) {
                    sh.found = threadIdx.x * kMine + i;
                    sh.before = w;
                    sh.weight = (u64)top_k - c;
                }
                c += count[i];
                w += mass[i];
            }
            __syncthreads();
            k_bin = (int)sh.found;
            in_front = sh.before;
            keep = (int)sh.weight;
            members = gather(n, [&](float x, int) { return bin_of<7>(__fsub_rn(big, x)) == k_bin; });
            if (members > kMembers) return false;
            for (int i = threadIdx.x; i < members; i += kSThreads) {
                const float x = sh.bin_x[i];
                const int at = sh.bin_index[i];
                int rank_in = 0;
                for (int k = 0; k < members; ++k) rank_in += ahead(sh.bin_x[k], sh.bin_index[k], x, at);
                if (rank_in < keep) atomicAdd(&sh.kept, weight(big, x));
                if (rank_in == keep - 1) {
                    sh.cut_x = x;
                    sh.cut_index = (uint32_t)at;
                }
            }
            __syncthreads();
            S = in_front + sh.kept;
        }
        if (top_p < 1.0f) {
            const u64 target = max(part_of(S, part31(top_p)), 1ull);
            if (target > all) return false;
            u64 w = pre_mass, front = in_front;
            if (target <= in_front) {  // in front of top-k's bin
                __syncthreads();       // (found and before have been read)
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    if (w < target && w + mass[i] >= target) {
                        sh.found = threadIdx.x * kMine + i;
                        sh.before = w;
                    }
                    w += mass[i];
                }
                __syncthreads();
                const int p_bin = (int)sh.found;
                front = sh.before;
                members = gather(n, [&](float x, int) { return bin_of<7>(__fsub_rn(big, x)) == p_bin; });
                if (members > kMembers) return false;
            }
            // (a token that top-k does not leave has all of what it leaves in front of it, which is no less than target)
            for (int i = threadIdx.x; i < members; i += kSThreads) {
                const float x = sh.bin_x[i];
                const int at = sh.bin_index[i];
                u64 before = front;
                for (int k = 0; k < members; ++k)
                    if (ahead(sh.bin_x[k], sh.bin_index[k], x, at)) before += weight(big, sh.bin_x[k]);
                if (before < target && before + weight(big, x) >= target) {
                    sh.cut_x = x;
                    sh.cut_index = (uint32_t)at;
                }
            }
            __syncthreads();
        }
        // Z and the choice, by bins of indexes
        const float cut_x = sh.cut_x;
        const uint32_t cut_index = sh.cut_index;
        auto kept = [&](float x, int i) {
            const u64 w = x > cut_x || (x == cut_x && (uint32_t)i <= cut_index) ? weight(big, x) : 0ull;
            return w >= least ? w : 0ull;
        };
        const int shift = max(0, 32 - __clz(a.j.V - 1) - 11);
        for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.bins[i] = 0;
        __syncthreads();
        listed(n, [&](float x, int i) {
            const u64 w = kept(x, i);
            if (w) atomicAdd(&sh.bins[i >> shift], w);
        });
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) mass[i] = sh.bins[threadIdx.x * kMine + i];
        u64 Z, w = scan(mass, sh.warp, Z);
        const u64 at_random = random_part(Z);
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            if (w <= at_random && w + mass[i] > at_random) {
                sh.found = threadIdx.x * kMine + i;
                sh.before = w;
            }
            w += mass[i];
        }
        __syncthreads();
        const int i_bin = (int)sh.found;
        const u64 front = sh.before;
        members = gather(n, [&](float x, int i) { return i >> shift == i_bin && kept(x, i) != 0; });
        if (members > kMembers) return false;
        for (int i = threadIdx.x; i < members; i += kSThreads) {
            const int at = sh.bin_index[i];
            u64 before = front;
            for (int k = 0; k < members; ++k)
                if (sh.bin_index[k] < at) before += weight(big, sh.bin_x[k]);
            const u64 mine = weight(big, sh.bin_x[i]);
            if (before <= at_random && before + mine > at_random) choose(at, mine, Z);
        }
        return true;
    }

    // With top-k or top-p.
    __device__ __forceinline__ void limited(int top_k, float top_p, u64 least, const float (&g)[kGroups]) {
        // The bin up to which so many groups have their largest value.
        const int most_k = ctas > 1 ? 2 * kMostK : kMostK;  // (the groups are 2048 a CTA)
        const uint32_t want = top_k ? (uint32_t)min(top_k, most_k) : (uint32_t)kTopPList;
        for (int i = threadIdx.x; i < kSThreads; i += kSThreads) sh.counts[i] = 0;
        if (threadIdx.x == 0) {
            sh.found = kSThreads - 1;
            sh.count = 0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
            const float d = __fsub_rn(big, g[i]);
            if (d < 64.0f) atomicAdd(&sh.counts[bin_of<5>(d)], 1u);
        }
        meet();
        static_assert(kSThreads == 16 << 5, "a bin a thread");
        uint32_t c = 0;
        for (uint32_t k = 0; k < ctas; ++k) c += ctas > 1 ? peer_u32(&sh.counts[threadIdx.x], k) : sh.counts[threadIdx.x];
        uint32_t pre = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(kFull, pre, o);
            if (lane >= o) pre += u;
        }
        if (lane == 31) sh.warp_count[warp] = pre;
        __syncthreads();
        pre -= c;
        for (int k = 0; k < warp; ++k) pre += sh.warp_count[k];
        if (pre < want && pre + c >= want) sh.found = threadIdx.x;
        __syncthreads();
        const float near = bin_end<5>((int)sh.found);
        auto collect = [&](float x, int i) {
            const uint32_t p = atomicAdd(&sh.count, 1u);
            if (p < (uint32_t)kList) {
                sh.x[p] = x;
                sh.index[p] = i;
            }
        };
        u64 total = 0;
        if (top_k)
            pass<false, true>(0, near, collect);
        else
            total = pass<true, true>(0, near, collect);
        if (!top_k) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(kFull, total, o);
            if (lane == 0) sh.warp[warp] = total;
            __syncthreads();
            total = 0;
#pragma unroll
            for (int k = 0; k < kSWarps; ++k) total += sh.warp[k];
            if (threadIdx.x == 0) sh.cta = total;
        }
        meet();
        uint32_t n = sh.count;
        bool fits = top_k <= most_k;
        if (ctas > 1) {
            n = 0;
            total = 0;
            for (uint32_t k = 0; k < ctas; ++k) {
                n += peer_u32(&sh.count, k);
                if (!top_k) total += peer_u64(&sh.cta, k);
            }
        }
        fits = fits && n <= (uint32_t)kList;
        if (rank == 0) {
            bool done = false;
            if (fits) {
                uint32_t at = sh.count;
                for (uint32_t k = 1; k < ctas; ++k) {
                    const uint32_t theirs = peer_u32(&sh.count, k);
                    for (uint32_t i = threadIdx.x; i < theirs; i += kSThreads) {
                        sh.x[at + i] = __uint_as_float(peer_u32(reinterpret_cast<const uint32_t *>(&sh.x[i]), k));
                        sh.index[at + i] = (int)peer_u32(reinterpret_cast<const uint32_t *>(&sh.index[i]), k);
                    }
                    at += theirs;
                }
                __syncthreads();
                done = choose_listed((int)n, top_k, top_p, least, total);
            }
            if (threadIdx.x == 0) sh.general = !done;
        }
        meet();
        const bool again = ctas > 1 ? peer_u32(&sh.general, 0) != 0 : sh.general != 0;
        meet();
        if (again) limits_by_digits(*this, top_k, top_p, least);
    }
};
// (A copy of the row: its values stay in the caller's registers.)
template <int kType>
__device__ void limits_by_digits(Row<kType> r, int top_k, float top_p, u64 least) {
    r.general(top_k, top_p, least);
}

template <int kType>
__global__ void __launch_bounds__(kSThreads, 2) k_sample(const __grid_constant__ SampleArgs a) {
    follow();
    extern __shared__ __align__(16) unsigned char s_mem[];
    SampleShared &sh = *reinterpret_cast<SampleShared *>(s_mem);
    const SampleJob &j = a.j;
    cluster_begin((uint32_t)a.ctas);
    Row<kType> r{a, sh};
    r.t = blockIdx.x / a.ctas;
    r.lane = threadIdx.x % 32;
    r.warp = threadIdx.x / 32;
    r.type = known<kType>(j.logits.type);
    r.ctas = (uint32_t)a.ctas;
    r.rank = blockIdx.x % (uint32_t)a.ctas;
    const int V = j.V;
    const char *row = static_cast<const char *>(row_of(j.logits, r.type, r.t));
    const int before16 = (int)(reinterpret_cast<uintptr_t>(row) % 16);
    r.base = row - before16;
    r.off = before16 / (two_bytes(r.type) ? 2 : 4);
    r.end = r.off + V;
    r.tiles = (r.end + kTile - 1) / kTile;
    r.share = (r.tiles + a.ctas * kSWarps - 1) / (a.ctas * kSWarps);
    r.begin = r.begin_of(r.warp);
    r.last = r.last_of(r.warp);
    r.allowed = j.allowed ? j.allowed + r.t * j.allowed_row : nullptr;

    const pvmvmd_sampling &how = j.how;
    const float temperature = how.temperature_dev ? how.temperature_dev[r.t] : how.temperature;
    const int top_k = how.top_k_dev ? how.top_k_dev[r.t] : how.top_k;
    const float top_p = how.top_p_dev ? how.top_p_dev[r.t] : how.top_p;
    const float min_p = how.min_p_dev ? how.min_p_dev[r.t] : how.min_p;
    const bool greedy = !(temperature > 0.0f);
    r.m = row_scale(j.logits, r.t);
    if (!greedy) {
        r.m = __fmul_rn(r.m, __fdiv_rn(1.442695041f, temperature));
        if (r.m > kFltMax) r.m = kFltMax;  // (NaN stays, and with it no token)
    }

    float g[kGroups];
    r.largest(g);
    uint32_t key = kNoKey;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) key = max(key, key_of(g[i]));
    cluster_begun(r.ctas);
    r.top = r.max_key(key);
    const bool writes = threadIdx.x == 0 && r.rank == 0;
    if (r.top <= kNoKey) {
        if (writes) {
            j.token[r.t] = -1;
            if (j.logprob) j.logprob[r.t] = -INFINITY;
        }
        return;
    }
    r.big = of_key(r.top);
    if (greedy) {  // the lowest index, as the largest of its complement
        uint32_t low = 0;
        if (__any_sync(kFull, key == r.top))
            r.each([&](float x, int i) {
                if (key_of(x) == r.top) low = max(low, ~(uint32_t)i);
            });
        low = ~r.max_key(low);
        if (writes) {
            j.token[r.t] = (int)low;
            if (j.logprob) j.logprob[r.t] = 0.0f;
        }
        return;
    }
    const u64 least = (u64)part31(min_p) << 9;
    const bool by_k = top_k >= 1 && top_k < V;
    if (by_k || top_p < 1.0f) {
        r.limited(by_k ? top_k : 0, top_p, least, g);
        return;
    }
    const u64 sum = r.template pass<true, false>(least, 0.0f, [](float, int) {});
    r.choose_in_order(sum, [&](float x, int) {
        const u64 w = weight(r.big, x);
        return w >= least ? w : 0ull;
    });
}

template <int kType>
cudaError_t launch_type(const SampleArgs &a, cudaStream_t s) {
    const cudaError_t e = func_attr(reinterpret_cast<const void *>(k_sample<kType>), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)sizeof(SampleShared));
    if (e != cudaSuccess) return e;
    return launch_cluster(k_sample<kType>, dim3((unsigned)(a.j.T * a.ctas)), a.ctas, kSThreads, sizeof(SampleShared), s, a);
}

}  // namespace

cudaError_t launch_sample(const SampleJob &j, cudaStream_t s) {
    SampleArgs a{j, 1};
    while (a.ctas < kMostCluster && (int64_t)j.T * a.ctas * 2 <= 304 && j.V / a.ctas >= 8192) a.ctas *= 2;
    if (j.allowed || j.logits.channel_scale_dev) return launch_type<kAny>(a, s);
    switch (j.logits.type) {
        case kBf16: return launch_type<kBf16>(a, s);
        case kF16: return launch_type<kF16>(a, s);
        case kF32: return launch_type<kF32>(a, s);
        default: return launch_type<kField>(a, s);
    }
}

}  // namespace pv
