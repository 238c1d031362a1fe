// The choice of the next token (pvmvmd_sample).
//
// A cluster of CTAs takes a row.  Weights are whole numbers, so their sums are the same in any
// order, and no result depends on the order of atomic operations or of a list.
//
// Without top-k and top-p a row is read twice: for the largest x, and for the weights' sum; then the warp's
// share where the choice falls is read once more.  The first reading waits for memory and the second for the pipe of products
// and sums, in turn in each CTA: over both, half of an SM's issue slots are used.
// With them, the threads' largest values, four a thread, say where about the k-th largest lies (there are at least k
// values above the k-th largest of them); the second reading puts the tokens up to there into a list, of a few
// times k, and the first CTA finds limits and choice in it: by histograms, whose one bin
// that a limit falls into is resolved by comparing its members with one another.
// Where the list does not hold what the limits leave (flat rows, a large k), a histogram of all tokens says in
// which bin a limit falls; that bin's tokens become the list, in which the limit is looked for digit by digit.
// Where they are too many for it (equal logits), the digits are those of all tokens, each another reading.
//
// 128000 logits a row: greedily 512 rows in 44 us (32 bits; 6.0 TB/s), whole distributions 113, top-k 50 74, top-p
// 0.5 139, flat rows with top-p 0.9 720; one row 3.9, 9.8, 10.9 and 16.8 us.
#include "rows.cuh"

namespace pv {
namespace {

constexpr int kSThreads = 512, kSWarps = kSThreads / 32;
constexpr int kBins = 2048;

constexpr int kList = 4096;      // tokens of the list
// A larger k (twice of it with several CTAs) is not looked for in a list.  (512 rows of 128000 with k 1000: 99 us from the
// list, 313 by histograms.  Up to 2000, k 1500 takes 124 in place of 321, but with 2000 the list overflows: 427 for 325.)
constexpr int kMostK = 1024;
constexpr int kMembers = 1024;   // of a bin at most that are compared with one another
// Tokens that are put in a list for top-p alone, about.  (With 384, 768 and 1536: 512 rows of 128000 with top-p 0.5 114, 127 and
// 193 us, 64 rows with 0.9 79, 74 and 70, 64 flat ones with 0.1 103, 105 and 44.)
constexpr int kTopPList = 768;
constexpr int kFew = 128;        // tokens of a list that are compared with one another at once
constexpr int kGroups = 4;       // largest values that a thread keeps
constexpr int kExchanges = 4;    // between the CTAs of a row, at most
using u64 = unsigned long long;

struct SampleSmall {  // what a row without top-k and top-p needs
    u64 warp[kSWarps], cta[kExchanges][kMostCluster];
    uint32_t warp_count[kSWarps];
};
struct SampleShared : SampleSmall {
    uint32_t low[kBins], high[kBins];  // bins' sums
    uint32_t counts[kBins];
    float x[kList], bin_x[kList];      // the list; one bin's members
    int index[kList], bin_index[kList];
    u64 before, weight, kept, few[kFew];
    uint32_t found, count, members, cut_index, general, bin;
    float cut_x;
};

__device__ __forceinline__ u64 peer_u64(const u64 *p, uint32_t rank) {
    uint32_t a;
    u64 v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void store_peer_u64(const u64 *p, uint32_t rank, u64 v) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}
__device__ __forceinline__ void store_peer_u32(const void *p, uint32_t rank, uint32_t v) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
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
// What is in bin b.
struct Range {
    uint32_t from, to;  // bits of distances, `to` not among them
};
template <int kFine>
__device__ __forceinline__ Range range_of(int b) {
    const uint32_t from = (uint32_t)(b + (117 << kFine)) << (23 - kFine);
    return Range{b ? from : 0u, from + (1u << (23 - kFine))};
}

struct SampleArgs {
    SampleJob j;
    int ctas;  // of a row
};

// Sums of 64 bits in shared memory, in two words: an addition of 32 bits is one instruction, one of
// 64 a loop, which equal tokens' bins make long.
__device__ __forceinline__ void add_to(SampleShared &sh, int bin, u64 w) {
    const uint32_t lo = (uint32_t)w, old = atomicAdd(&sh.low[bin], lo);
    const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old);
    if (hi) atomicAdd(&sh.high[bin], hi);
}
__device__ __forceinline__ u64 sum_of(const SampleShared &sh, int bin) { return (u64)sh.high[bin] << 32 | sh.low[bin]; }

struct RowData {
    const SampleArgs &a;
    SampleShared &sh;
    int64_t t;
    int lane, warp, type;
    uint32_t rank, ctas;
    const char *base;  // the 16-byte boundary at or before the row
    int off, end;      // the row's tokens are off .. end - 1 from there
    int tiles, share;  // the row's, and a warp's
    int begin, last;   // tiles of this warp
    float m;
    const uint32_t *allowed;
    bool wide_scales;  // channel scales can be read four at a time
    int exchanges;     // so far
    float big;         // the largest x
    uint32_t top;      // its key
};
__device__ __noinline__ void limits_in_all(RowData r, int top_k, float top_p, u64 least);
__device__ __noinline__ bool choose_from_list(RowData r, int n, int top_k, float top_p, u64 least, u64 total);

// kType: the logits', or any.
template <int kType>
struct Row : RowData {
    __device__ __forceinline__ void meet() const {
        if (ctas > 1)
            clusters_meet();
        else
            __syncthreads();
    }
    // Of tiles begin .. last - 1 those that lie in the row whole: from .. to - 1 (from <= to).
    __device__ __forceinline__ int whole_from(int begin, int last) const { return min(last, max(begin, (off + kTile - 1) / kTile)); }
    __device__ __forceinline__ int whole_to(int begin, int last) const {
        return max(whole_from(begin, last), min(last, end / kTile));
    }
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
        if (allowed) {
            const int w = i0 >> 5, words = (V + 31) >> 5;
            const uint32_t lo = w >= 0 && w < words ? allowed[w] : 0u;
            const uint32_t hi = (i0 & 31) > 24 && w + 1 < words ? allowed[w + 1] : 0u;
            ok = __funnelshift_r(lo, hi, i0 & 31);
        }
#pragma unroll
        for (int e = 0; e < kWide; ++e) {
            float v = __fmul_rn(e & 1 ? second(v2[e / 2]) : first(v2[e / 2]), m);
            const bool in = i0 + e >= 0 && i0 + e < V;
            if (l.channel_scale_dev && in) v = __fmul_rn(v, l.channel_scale_dev[i0 + e]);
            v = v > -INFINITY ? fminf(v, kFltMax) : -INFINITY;  // (NaN is not)
            x[e] = in && (ok >> e & 1) ? v : -INFINITY;
        }
        return i0;
    }
    // Bit e: whether the token i0 + e may be chosen, for a tile inside the row.
    __device__ __forceinline__ uint32_t allowed_bits(int i0) const {
        const int w = i0 >> 5;
        return __funnelshift_r(allowed[w], (i0 & 31) > 24 ? allowed[w + 1] : 0u, i0 & 31);
    }
    // The same for a tile inside the row, from what load_inside gave, without the cut at FLT_MAX: NaN and
    // infinities as they come.
    __device__ __forceinline__ void plain_tokens(const Raw &r, int i0, Two (&x)[kTwos]) const {
        unpack(r, type, x);
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = mul2(x[i], both(m));
        if (const float *c = a.j.logits.channel_scale_dev) {
            Raw s;
            if (wide_scales) {
                s.a = *reinterpret_cast<const uint4 *>(c + i0);
                s.b = *reinterpret_cast<const uint4 *>(c + i0 + 4);
            } else {
                const uint32_t *p = reinterpret_cast<const uint32_t *>(c + i0);
                s.a = make_uint4(p[0], p[1], p[2], p[3]);
                s.b = make_uint4(p[4], p[5], p[6], p[7]);
            }
            Two v[kTwos];
            unpack(s, PVMVMD_F32, v);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[i] = mul2(x[i], v[i]);
        }
        if (allowed) {
            const uint32_t ok = allowed_bits(i0);
#pragma unroll
            for (int i = 0; i < kTwos; ++i)
                x[i] = two(ok >> 2 * i & 1 ? first(x[i]) : -INFINITY, ok >> (2 * i + 1) & 1 ? second(x[i]) : -INFINITY);
        }
    }
    __device__ __forceinline__ int index_of(int tile) const { return tile * kTile + lane * kWide - off; }

    // f(x, index) for every token of tiles from .. to - 1 that may be chosen
    template <typename F>
    __device__ __forceinline__ void each(int from, int to, F f) const {
#pragma unroll 1
        for (int k = from; k < to; ++k) {
            float x[kWide];
            const int i0 = tokens(k, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e)
                if (x[e] > -INFINITY) f(x[e], i0 + e);
        }
    }

    __device__ __forceinline__ u64 peer_sum(int bin, uint32_t c) const {
        return (u64)peer_u32(&sh.high[bin], c) << 32 | peer_u32(&sh.low[bin], c);
    }
    // Every CTA's value, in this CTA's memory.
    __device__ __forceinline__ const u64 *exchange(u64 v) {
        u64 *all = sh.cta[exchanges++];
        if (ctas > 1) {
            if (threadIdx.x < ctas) store_peer_u64(&all[rank], threadIdx.x, v);
            clusters_meet();
        } else {
            if (threadIdx.x == 0) all[0] = v;
            __syncthreads();
        }
        return all;
    }
    // The largest key of all CTAs, and the first of them that has it.
    __device__ __forceinline__ uint32_t max_key(uint32_t k, int &owner) {
        k = __reduce_max_sync(kFull, k);
        if (lane == 0) sh.warp_count[warp] = k;
        __syncthreads();
        k = __reduce_max_sync(kFull, lane < kSWarps ? sh.warp_count[lane] : 0u);
        owner = 0;
        if (ctas == 1) return k;
        const u64 *all = exchange(k);
        const uint32_t theirs = lane < (int)ctas ? (uint32_t)all[lane] : 0u;
        k = __reduce_max_sync(kFull, theirs);
        owner = __ffs(__ballot_sync(kFull, lane < (int)ctas && theirs == k)) - 1;
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
        const int from = whole_from(begin, last), to = whole_to(begin, last);
        for (; k < from; ++k) edge(k);
        if (m > 0.0f && !allowed && !a.j.logits.channel_scale_dev) {
            // rounding keeps the order, so that the largest logit has the largest x
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
        } else {
#pragma unroll 2
            for (; k < to; ++k) {
                Two x[kTwos];
                plain_tokens(load_inside(k), index_of(k), x);
#pragma unroll
                for (int i = 0; i < kTwos; ++i) {  // (NaN is not taken)
                    g[i] = fmaxf(g[i], fminf(fmaxf(first(x[i]), -INFINITY), kFltMax));
                    g[i] = fmaxf(g[i], fminf(fmaxf(second(x[i]), -INFINITY), kFltMax));
                }
            }
        }
#pragma unroll 1
        for (; k < last; ++k) edge(k);
    }

    // One pass over tiles begin .. last - 1: the sum, where asked for, of the weights that are at least `least` (and with kCut of
    // tokens up to a cut); collect(x, index) for the tokens whose distance is below `near`; hist(d, w) for all of some weight.
    struct Cut {
        float x;
        uint32_t index;
        __device__ __forceinline__ bool keeps(float v, int i) const { return v > x || (v == x && (uint32_t)i <= index); }
    };
    // kLeast: `least` may be above 0.
    // kSparse: few tokens are collected.
    template <bool kSum, bool kCollect, bool kHist, bool kCut, bool kLeast, bool kSparse = false, typename C, typename H>
    __device__ __forceinline__ u64 pass(int begin, int last, u64 least, float near, Cut cut, C collect, H hist) const {
        u64 sum = 0;
        int k;
        auto edge = [&](int tile) {
            float x[kWide];
            const int i0 = tokens(tile, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e) {
                if (x[e] > -INFINITY) {
                    if (kSum && (!kCut || cut.keeps(x[e], i0 + e))) {
                        const u64 w = weight(big, x[e]);
                        sum += w >= least ? w : 0ull;
                    }
                    const float d = __fsub_rn(big, x[e]);
                    if (kCollect && d < near) collect(x[e], i0 + e);
                    if (kHist) hist(d, weight(big, x[e]));
                }
            }
        };
        const int from = whole_from(begin, last), to = big < kFltMax ? whole_to(begin, last) : from;  // (else x may be cut)
#pragma unroll 1
        for (k = last - 1; k >= to; --k) edge(k);
        // Backwards: the cache still has what was read last.  The next two tiles are on their way meanwhile.
        Raw tile0, tile1;
        if (k >= from) {
            tile0 = load_inside(k);
            tile1 = load_inside(max(k - 1, from));
        }
#pragma unroll 2
        for (; k >= from; --k) {
            Two x[kTwos];
            const int i0 = index_of(k);
            const Raw now = tile0;
            tile0 = tile1;
            tile1 = load_inside(max(k - 2, from));
            plain_tokens(now, i0, x);
            uint32_t hits = 0, low = 0;
#pragma unroll
            for (int i = 0; i < kTwos; ++i) {
                Two d = sub2(both(big), x[i]);
                if (kCollect) hits |= (first(d) < near ? 1u << 2 * i : 0u) | (second(d) < near ? 2u << 2 * i : 0u);
                if (kSum || kHist) {
                    d = two(fminf(first(d), 63.0f), fminf(second(d), 63.0f));  // (NaN: 63)
                    Two n;
                    const Two r = add2(exp_poly(split(d, n), 4194304.0f), both(8388608.0f));
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t p = (uint32_t)(h ? r.v >> 32 : r.v) & 0x7fffffu;
                        const uint32_t q = (uint32_t)(h ? n.v >> 32 : n.v);
                        if (kCut && !cut.keeps(h ? second(x[i]) : first(x[i]), i0 + 2 * i + h)) p = 0;
                        if (kHist || kLeast) {
                            const u64 w = ((u64)p << 18) >> (q - 0x4b400000u);
                            if (kHist)
                                hist(h ? second(d) : first(d), w);
                            else
                                sum += w >= least ? w : 0ull;
                        } else {
                            // p 2^(18 - n) for n < 18, a product that is added in one instruction; the others are below 2^23
                            sum += (u64)p * shift_left(2u, 0x4b400000u + 17u - q);
                            low += shift_right(p, q - (0x4b400000u + 18u));
                        }
                    }
                }
            }
            if (kSum) sum += low;
            if (kSparse) {  // (most tiles have none)
#pragma unroll 1
                while (hits) {
                    const int e = __ffs(hits) - 1;
                    const Two v = e & 4 ? (e & 2 ? x[3] : x[2]) : (e & 2 ? x[1] : x[0]);
                    collect(e & 1 ? second(v) : first(v), i0 + e);
                    hits &= hits - 1;
                }
            }
            if (kCollect && !kSparse && hits) {
#pragma unroll
                for (int e = 0; e < kWide; ++e)
                    if (hits >> e & 1) collect(e & 1 ? second(x[e / 2]) : first(x[e / 2]), i0 + e);
            }
        }
#pragma unroll 1
        for (; k >= begin; --k) edge(k);
        return sum;
    }
    __device__ __forceinline__ Cut no_cut() const { return Cut{-INFINITY, ~0u}; }

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
            for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.low[i] = sh.high[i] = 0;
            if (threadIdx.x == 0) sh.found = ~0u;
            __syncthreads();
            const uint32_t high = v;
            each(begin, last, [&](float x, int i) {
                uint32_t value;
                u64 w;
                if (f(x, i, value, w) && ((u64)value >> left) == ((u64)high >> left) && w)
                    add_to(sh, (int)((value >> open) & ((1u << digit) - 1)), w);
            });
            meet();
            constexpr int kMine = kBins / kSThreads;
            u64 mine[kMine], total;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int b = (int)threadIdx.x * kMine + i;
                mine[i] = 0;
                for (uint32_t c = 0; c < ctas; ++c) mine[i] += ctas > 1 ? peer_sum(b, c) : sum_of(sh, b);
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

    // The lowest index of the largest x, in the first CTA that has it: all warps look at the tiles of the first warp that
    // has it.
    __device__ __forceinline__ void first_largest() const {
        const int w = __ffs(__ballot_sync(kFull, lane < kSWarps && sh.warp_count[lane % kSWarps] == top)) - 1;
        const int per = (last_of(w) - begin_of(w) + kSWarps - 1) / kSWarps;
        const int from = min(last_of(w), begin_of(w) + warp * per), to = min(last_of(w), from + per);
        uint32_t low = ~0u;
        for (int k = from; k < to; ++k) {
            float x[kWide];
            const int i0 = tokens(k, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e)
                if (x[e] > -INFINITY && key_of(x[e]) == top) low = min(low, (uint32_t)(i0 + e));
        }
        low = __reduce_min_sync(kFull, low);
        if (lane == 0) sh.warp[warp] = low;
        __syncthreads();
        if (warp == 0) {
            low = __reduce_min_sync(kFull, lane < kSWarps ? (uint32_t)sh.warp[lane] : ~0u);
            if (lane == 0) {
                a.j.token[t] = (int)low;
                if (a.j.logprob) a.j.logprob[t] = 0.0f;
            }
        }
    }

    // The choice among the tokens that kept(x, index) gives a weight to; sum_of_tiles(begin, last): what those of a warp's
    // tiles weigh.
    template <typename F, typename G>
    __device__ __forceinline__ void choose_in_order(F kept, G sum_of_tiles) {
        auto warp_sum = [&](int from, int to) {
            u64 sum = sum_of_tiles(from, to);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
            __syncthreads();  // (earlier ones have been read)
            if (lane == 0) sh.warp[warp] = sum;
            __syncthreads();
            return sum;
        };
        warp_sum(begin, last);
        u64 mine = 0, front = 0, Z = 0;  // of this CTA; of the CTAs in front; of all
#pragma unroll
        for (int k = 0; k < kSWarps; ++k) mine += sh.warp[k];
        const u64 *all = exchange(mine);
        for (uint32_t c = 0; c < ctas; ++c) {
            if (c < rank) front += all[c];
            Z += all[c];
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
        const u64 part = warp_sum(from, to);
        for (int k = 0; k < warp; ++k) front += sh.warp[k];
        if (at < front || at >= front + part) return;
#pragma unroll 1
        for (int k = from; k < to; ++k) {
            float x[kWide];
            u64 w[kWide], all = 0;
            const int i0 = tokens(k, x);
#pragma unroll
            for (int e = 0; e < kWide; ++e) all += w[e] = x[e] > -INFINITY ? kept(x[e], i0 + e) : 0ull;
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
        choose_in_order(kept, [&](int from, int to) {
            u64 sum = 0;
            each(from, to, [&](float x, int i) { sum += kept(x, i); });
            return sum;
        });
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

    // The same from a list of at most kFew tokens, a thread each, which compare themselves with all others: four
    // barriers instead of fifteen.  (One row of 128000 logits with top-k 50 and top-p 16.1 us through the bins, 13.8 so; lists of
    // 230 take 8 us longer so.)
    __device__ __forceinline__ bool choose_few(int n, int top_k, float top_p, u64 least, u64 total) {
        const int i = threadIdx.x;
        const bool mine = i < n;
        const float x = mine ? sh.x[i] : 0.0f;
        const int at = mine ? sh.index[i] : 0;
        const u64 w = mine ? weight(big, x) : 0ull;
        if (mine) sh.few[i] = w;
        __syncthreads();
        int place = 0;  // in falling order
        u64 before = 0, all = 0;
        if (i < (n + 31) / 32 * 32) {
#pragma unroll 4
            for (int k = 0; k < n; ++k) {
                const u64 v = sh.few[k];
                const bool front = ahead(sh.x[k], sh.index[k], x, at);
                place += front;
                before += front ? v : 0ull;
                all += v;
            }
        }
        const int last = top_k && top_k < n ? top_k - 1 : n - 1;
        if (mine && place == last) sh.kept = before + w;
        if (i == 0) sh.weight = all;
        __syncthreads();
        bool keep = mine && place <= last;
        if (top_p < 1.0f) {
            const u64 part = part_of(total ? total : sh.kept, part31(top_p));
            if (part > sh.weight) return false;
            keep = keep && (place == 0 || before < part);
        }
        keep = keep && w >= least;
        __syncthreads();  // (what the weights are read for is done)
        if (mine) sh.few[i] = keep ? w : 0ull;
        __syncthreads();
        if (i < (n + 31) / 32 * 32) {
            u64 front = 0, Z = 0;
#pragma unroll 4
            for (int k = 0; k < n; ++k) {
                const u64 v = sh.few[k];
                front += sh.index[k] < at ? v : 0ull;
                Z += v;
            }
            const u64 at_random = random_part(Z);
            if (keep && front <= at_random && front + w > at_random) choose(at, w, Z);
        }
        return true;
    }
    // The choice from a list of n tokens, which are all those nearer than the first one that is not there.  total: what
    // all tokens of the row weigh, 0 where top_k limits them.  False where the limits leave more than the list, or
    // too many fall into one bin.
    __device__ __forceinline__ bool choose_listed(int n, int top_k, float top_p, u64 least, u64 total) {
        if (n <= kFew) return choose_few(n, top_k, top_p, least, total);
        constexpr int kMine = kBins / kSThreads;
        for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.low[i] = sh.high[i] = sh.counts[i] = 0;
        if (threadIdx.x == 0) {
            sh.found = ~0u;
            sh.cut_x = -INFINITY;
            sh.cut_index = ~0u;
            sh.kept = 0;
        }
        __syncthreads();
        listed(n, [&](float x, int) {
            const int b = bin_of<7>(__fsub_rn(big, x));
            add_to(sh, b, weight(big, x));
            atomicAdd(&sh.counts[b], 1u);
        });
        __syncthreads();
        u64 mass[kMine], all;
        uint32_t count[kMine], number;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            mass[i] = sum_of(sh, threadIdx.x * kMine + i);
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
        for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.low[i] = sh.high[i] = 0;
        __syncthreads();
        listed(n, [&](float x, int i) {
            const u64 w = kept(x, i);
            if (w) add_to(sh, i >> shift, w);
        });
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) mass[i] = sum_of(sh, threadIdx.x * kMine + i);
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

    // The tokens whose distance's bits are in a range, to this CTA's part of the list; then, in the first CTA, all of
    // them.  Their number, in every CTA; what is above kList is not in the list.  total: of the row's weights, where
    // asked for.
    template <bool kSum, bool kSparse = false>
    __device__ __forceinline__ uint32_t collect_list(Range range, u64 &total) {
        if (threadIdx.x == 0) sh.count = 0;
        __syncthreads();
        auto collect = [&](float x, int i) {
            if (range.from && __float_as_uint(__fsub_rn(big, x)) < range.from) return;
            const uint32_t p = atomicAdd(&sh.count, 1u);
            if (p < (uint32_t)kList) {
                sh.x[p] = x;
                sh.index[p] = i;
            }
        };
        total = pass<kSum, true, false, false, false, kSparse>(begin, last, 0, __uint_as_float(range.to), no_cut(), collect,
                                                               [](float, u64) {});
        if (kSum) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(kFull, total, o);
            if (lane == 0) sh.warp[warp] = total;
        }
        __syncthreads();
        total = 0;
        if (kSum)
#pragma unroll
            for (int k = 0; k < kSWarps; ++k) total += sh.warp[k];
        uint32_t n = sh.count;
        if (ctas == 1) return n;
        const uint32_t mine = min(n, (uint32_t)kList + 1);
        const u64 *all = exchange(mine);
        n = 0;
        for (uint32_t c = 0; c < ctas; ++c) n += (uint32_t)all[c];
        if (kSum) {
            const u64 *sums = exchange(total);
            total = 0;
            for (uint32_t c = 0; c < ctas; ++c) total += sums[c];
        }
        if (rank && n <= (uint32_t)kList) {
            uint32_t at = 0;
            for (uint32_t c = 0; c < rank; ++c) at += (uint32_t)all[c];
            for (uint32_t i = threadIdx.x; i < mine; i += kSThreads) {
                store_peer_u32(&sh.x[at + i], 0, __float_as_uint(sh.x[i]));
                store_peer_u32(&sh.index[at + i], 0, (uint32_t)sh.index[i]);
            }
        }
        clusters_meet();
        return n;
    }

    // The same as reach, for the first n tokens of the list and by one CTA.
    template <typename F>
    __device__ __forceinline__ bool reach_listed(int n, int bits, u64 target, F f, uint32_t &v, u64 &before, u64 &at) const {
        v = 0;
        before = at = 0;
        uint32_t open = 0;
        for (int left = bits; left > 0; left = (int)open) {
            const int digit = min(left, 11);
            open = (uint32_t)(left - digit);
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.low[i] = sh.high[i] = 0;
            if (threadIdx.x == 0) sh.found = ~0u;
            __syncthreads();
            const uint32_t high = v;
            listed(n, [&](float x, int i) {
                uint32_t value;
                u64 w;
                if (f(x, i, value, w) && ((u64)value >> left) == ((u64)high >> left) && w)
                    add_to(sh, (int)((value >> open) & ((1u << digit) - 1)), w);
            });
            __syncthreads();
            constexpr int kMine = kBins / kSThreads;
            u64 mine[kMine], total;
#pragma unroll
            for (int i = 0; i < kMine; ++i) mine[i] = sum_of(sh, threadIdx.x * kMine + i);
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
            __syncthreads();
            if (sh.found == ~0u) return false;
            v |= sh.found << open;
            before = sh.before;
            at = sh.weight;
        }
        return true;
    }
    // Of the listed tokens that `within` keeps, in order: those up to which `target` of weight lies (one each where
    // ones).  The cut after them.
    __device__ __forceinline__ Cut cut_listed(int n, u64 target, bool ones, Cut within) const {
        if (n <= kFew) {  // a thread each, which compares its token with all others
            const int i = threadIdx.x;
            const bool mine = i < n && within.keeps(sh.x[i], sh.index[i]);
            const float x = i < n ? sh.x[i] : 0.0f;
            const int at = i < n ? sh.index[i] : 0;
            const u64 w = !mine ? 0ull : ones ? 1ull : weight(big, x);
            if (i < n) sh.few[i] = w;
            __syncthreads();
            u64 before = 0;
            if (i < (n + 31) / 32 * 32)
#pragma unroll 4
                for (int k = 0; k < n; ++k) before += ahead(sh.x[k], sh.index[k], x, at) ? sh.few[k] : 0ull;
            if (mine && before < target && before + w >= target) {
                sh.cut_x = x;
                sh.cut_index = (uint32_t)at;
            }
            __syncthreads();
            return Cut{sh.cut_x, sh.cut_index};
        }
        uint32_t v;
        u64 before, at;
        reach_listed(n, 32, target, [&](float x, int i, uint32_t &value, u64 &w) {
            value = top - key_of(x);
            w = ones ? 1ull : weight(big, x);
            return within.keeps(x, i);
        }, v, before, at);
        const float x0 = of_key(top - v);
        const u64 each = ones ? 1ull : weight(big, x0), ties = (target - before + each - 1) / each;
        Cut cut{x0, x0 == within.x ? within.index : ~0u};
        if (ties < at / each) {
            u64 b, w1;
            reach_listed(n, 24, ties, [&](float x, int i, uint32_t &value, u64 &w) {
                value = (uint32_t)i;
                w = 1;
                return x == x0 && within.keeps(x, i);
            }, cut.index, b, w1);
        }
        return cut;
    }

    // A histogram of the tokens in a range, by bin(bits of the distance): weights, and numbers where asked for.  A
    // thread's bins of it, for all CTAs, and what lies in front of them.
    static constexpr int kMine = kBins / kSThreads;
    template <typename F>
    __device__ __forceinline__ void histogram(Range range, bool numbers, F bin, u64 (&mass)[kMine], u64 &pre_mass, u64 &all,
                                              uint32_t (&count)[kMine], uint32_t &pre_count, uint32_t &number) {
        for (int i = threadIdx.x; i < kBins; i += kSThreads) sh.low[i] = sh.high[i] = sh.counts[i] = 0;
        __syncthreads();
        pass<false, false, true, false, false>(begin, last, 0, 0.0f, no_cut(), [](float, int) {}, [&](float d, u64 w) {
            const uint32_t bits = __float_as_uint(d);
            if (w && bits >= range.from && bits < range.to) {
                const int b = bin(d, bits);
                add_to(sh, b, w);
                if (numbers) atomicAdd(&sh.counts[b], 1u);
            }
        });
        meet();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int b = threadIdx.x * kMine + i;
            mass[i] = sum_of(sh, b);
            count[i] = sh.counts[b];
            if (ctas > 1) {
                mass[i] = 0;
                count[i] = 0;
                for (uint32_t c = 0; c < ctas; ++c) {
                    mass[i] += peer_sum(b, c);
                    count[i] += peer_u32(&sh.counts[b], c);
                }
            }
        }
        pre_count = scan(count, sh.warp_count, number);
        pre_mass = scan(mass, sh.warp, all);
        meet();  // (the bins have been read)
    }
    // Where a limit falls: the bin, and what is in front of it.
    struct Fall {
        Range range;
        u64 mass;   // of weight
        u64 count;  // of tokens
    };
    // `target` of weight (by_count: of tokens) reached in a thread's bins: to shared memory.
    __device__ __forceinline__ int fall(bool by_count, u64 target, const u64 (&mass)[kMine], u64 pre_mass,
                                        const uint32_t (&count)[kMine], uint32_t pre_count, Fall &f) const {
        __syncthreads();  // (an earlier one's results have been read)
        u64 c = f.count + pre_count, w = f.mass + pre_mass;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const u64 v = by_count ? c : w;
            c += count[i];
            w += mass[i];
            if (v < target && (by_count ? c : w) >= target) {
                sh.bin = threadIdx.x * kMine + i;
                sh.before = w - mass[i];
                sh.weight = c - count[i];
            }
        }
        __syncthreads();
        f.mass = sh.before;
        f.count = sh.weight;
        return (int)sh.bin;
    }
    // The bin's tokens in the list, from narrower bins where they are too many; their number, or more than kList where
    // that does not help.
    __device__ __forceinline__ uint32_t narrow(bool by_count, u64 target, Fall &f) {
        u64 none;
        for (;;) {
            exchanges = 0;
            meet();  // (what it overwrites has been read)
            const uint32_t n = collect_list<false>(f.range, none), width = f.range.to - f.range.from;
            if (n <= (uint32_t)kList || width <= 1) return n;
            const int shift = max(0, 32 - __clz(width - 1) - 11);
            u64 mass[kMine], pre_mass, all;
            uint32_t count[kMine], pre_count, number;
            const uint32_t from = f.range.from;
            histogram(f.range, true, [&](float, uint32_t bits) { return (int)((bits - from) >> shift); }, mass, pre_mass, all, count,
                      pre_count, number);
            const uint32_t b = (uint32_t)fall(by_count, target, mass, pre_mass, count, pre_count, f);
            f.range = Range{from + (b << shift), min(f.range.to, from + ((b + 1) << shift))};
        }
    }

    // The limits looked for by histograms of all tokens.  False where equal distances have more of them than the list.
    __device__ __forceinline__ bool by_bins(int top_k, float top_p, u64 least) {
        u64 mass[kMine], pre_mass, all;
        uint32_t count[kMine], pre_count, number;
        histogram(Range{0, range_of<7>(kBins - 1).to}, top_k != 0, [](float d, uint32_t) { return bin_of<7>(d); }, mass, pre_mass,
                  all, count, pre_count, number);
        Cut cut = no_cut();
        u64 S = all;
        Fall f{Range{0, 0}, ~0ull, 0};  // of top-k: everything is in front of it where there is none
        uint32_t n = 0;
        if (top_k && (uint32_t)top_k < number) {
            f.mass = 0;
            f.range = range_of<7>(fall(true, (u64)top_k, mass, pre_mass, count, pre_count, f));
            n = narrow(true, (u64)top_k, f);
            if (n > (uint32_t)kList) return false;
            if (rank == 0) {
                cut = cut_listed((int)n, (u64)top_k - f.count, true, no_cut());
                if (threadIdx.x == 0) sh.kept = 0;
                __syncthreads();
                u64 mine = 0;
                listed((int)n, [&](float x, int i) { mine += cut.keeps(x, i) ? weight(big, x) : 0ull; });
                if (mine) atomicAdd(&sh.kept, mine);
                __syncthreads();
            }
            S = f.mass + (ctas > 1 ? (meet(), peer_u64(&sh.kept, 0)) : sh.kept);
        }
        if (top_p < 1.0f) {
            const u64 target = max(part_of(S, part31(top_p)), 1ull);
            if (target <= f.mass) {  // in front of top-k's bin, or without it
                f = Fall{Range{0, 0}, 0, 0};
                f.range = range_of<7>(fall(false, target, mass, pre_mass, count, pre_count, f));
                cut = no_cut();
                n = narrow(false, target, f);
                if (n > (uint32_t)kList) return false;
            }
            if (rank == 0) cut = cut_listed((int)n, target - f.mass, false, cut);
        }
        if (ctas > 1) {  // the first CTA's cut
            if (rank == 0 && threadIdx.x == 0) sh.cut_x = cut.x, sh.cut_index = cut.index;
            meet();
            cut = Cut{__uint_as_float(peer_u32(reinterpret_cast<const uint32_t *>(&sh.cut_x), 0)), peer_u32(&sh.cut_index, 0)};
        }
        exchanges = 0;
        meet();
        choose_in_order(
            [&](float x, int i) {
                const u64 w = cut.keeps(x, i) ? weight(big, x) : 0ull;
                return w >= least ? w : 0ull;
            },
            [&](int from, int to) {
                return pass<true, false, false, true, true>(from, to, least, 0.0f, cut, [](float, int) {}, [](float, u64) {});
            });
        return true;
    }

    // With top-k or top-p.
    __device__ __forceinline__ void limited(int top_k, float top_p, u64 least, const float (&g)[kGroups]) {
        // The bin up to which so many groups have their largest value.
        const int most_k = ctas > 1 ? 2 * kMostK : kMostK;  // (the groups are 2048 a CTA)
        const uint32_t want = top_k ? (uint32_t)min(top_k, most_k) : (uint32_t)kTopPList;
        bool again = top_k > most_k;
        if (!again) {
            sh.counts[threadIdx.x] = 0;
            if (threadIdx.x == 0) sh.found = kSThreads - 1;
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
            const Range near{0, range_of<5>((int)sh.found).to};
            u64 total = 0;
            const uint32_t n = top_k ? collect_list<false, true>(near, total) : collect_list<true>(near, total);
            again = n > (uint32_t)kList;
            if (!again) {
                if (rank == 0) {
                    const bool done = choose_from_list(*this, (int)n, top_k, top_p, least, total);
                    if (threadIdx.x < ctas) {
                        if (ctas > 1)
                            store_peer_u32(&sh.general, threadIdx.x, !done);
                        else
                            sh.general = !done;
                    }
                }
                meet();
                again = sh.general != 0;
            }
        }
        if (again) limits_in_all(*this, top_k, top_p, least);
    }
};
// (Copies of the row: its values stay in the caller's registers.)
__device__ bool choose_from_list(RowData d, int n, int top_k, float top_p, u64 least, u64 total) {
    return Row<kAny>{d}.choose_listed(n, top_k, top_p, least, total);
}
__device__ void limits_in_all(RowData d, int top_k, float top_p, u64 least) {
    Row<kAny> r{d};
    r.exchanges = 0;
    if (!r.by_bins(top_k, top_p, least)) {
        r.exchanges = 0;
        r.meet();
        r.general(top_k, top_p, least);
    }
}

// kLimited: rows may have top-k or top-p.  (Without them a third CTA an SM would find room, of 40 registers a thread; 512
// rows of 128000 take 122 us so, 113 with two.)
template <int kType, bool kLimited>
__global__ void __launch_bounds__(kSThreads, 2) k_sample(const __grid_constant__ SampleArgs a) {
    follow();
    extern __shared__ __align__(16) unsigned char s_mem[];
    SampleShared &sh = *reinterpret_cast<SampleShared *>(s_mem);
    const SampleJob &j = a.j;
    cluster_begin((uint32_t)a.ctas);
    Row<kType> r{RowData{a, sh}};
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
    r.wide_scales = r.off % 4 == 0 && reinterpret_cast<uintptr_t>(j.logits.channel_scale_dev) % 16 == 0;
    r.exchanges = 0;

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
    int owner;
    r.top = r.max_key(key, owner);
    const bool writes = threadIdx.x == 0 && r.rank == 0;
    if (r.top <= kNoKey) {
        if (writes) {
            j.token[r.t] = -1;
            if (j.logprob) j.logprob[r.t] = -INFINITY;
        }
        return;
    }
    r.big = of_key(r.top);
    if (greedy) {
        if ((int)r.rank == owner) r.first_largest();
        return;
    }
    const u64 least = (u64)part31(min_p) << 9;
    const bool by_k = top_k >= 1 && top_k < V;
    if (kLimited && (by_k || top_p < 1.0f)) {
        r.limited(by_k ? top_k : 0, top_p, least, g);
        return;
    }
    auto none = [](float, int) {};
    auto no_bin = [](float, u64) {};
    auto kept = [&](float x, int) {
        const u64 w = weight(r.big, x);
        return w >= least ? w : 0ull;
    };
    r.choose_in_order(kept, [&](int from, int to) {
        return least ? r.template pass<true, false, false, false, true>(from, to, least, 0.0f, r.no_cut(), none, no_bin)
                     : r.template pass<true, false, false, false, false>(from, to, 0, 0.0f, r.no_cut(), none, no_bin);
    });
}

template <int kType, bool kLimited>
cudaError_t launch_limited(const SampleArgs &a, cudaStream_t s) {
    const size_t smem = kLimited ? sizeof(SampleShared) : sizeof(SampleSmall);
    const cudaError_t e = func_attr(reinterpret_cast<const void *>(k_sample<kType, kLimited>),
                                    cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_cluster(k_sample<kType, kLimited>, dim3((unsigned)(a.j.T * a.ctas)), a.ctas, kSThreads, smem, s, a);
}
template <int kType>
cudaError_t launch_type(const SampleArgs &a, cudaStream_t s) {
    const pvmvmd_sampling &how = a.j.how;
    const bool by_k = how.top_k_dev || (how.top_k >= 1 && how.top_k < a.j.V), by_p = how.top_p_dev || how.top_p < 1.0f;
    return by_k || by_p ? launch_limited<kType, true>(a, s) : launch_limited<kType, false>(a, s);
}

}  // namespace

cudaError_t launch_sample(const SampleJob &j, cudaStream_t s) {
    // A row over as many CTAs as leave two an SM, of which each halving leaves 3000 tokens at least (one row of 128000 with
    // top-k and top-p 35 us by one CTA, 23, 16 and 13 by 2, 4 and 8; of 12000 8.9, 8.8 and 9.1 by 2, 4 and 8; of 6000 6.9
    // by one and 8.5 by two; 512 rows of 128000 119 by one each, 121 by two, 135 by four).  Clusters of 8 do not find
    // that many places: with 35 to 38 rows some wait for others (37 of 32001 19 us, 10.2 by clusters of 4; 32 11.2).
    SampleArgs a{j, 1};
    while (a.ctas < kMostCluster && (int64_t)j.T * a.ctas * 2 <= 2 * kSms && j.V / a.ctas >= 6000) a.ctas *= 2;
    switch (j.logits.type) {
        case kBf16: return launch_type<kBf16>(a, s);
        case kF16: return launch_type<kF16>(a, s);
        case kF32: return launch_type<kF32>(a, s);
        default: return launch_type<kField>(a, s);
    }
}

}  // namespace pv
