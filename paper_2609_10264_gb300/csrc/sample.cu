// The choice of the next token (pvmvmd_sample).
//
// A cluster of CTAs takes a row.  Weights are whole numbers, so their sums are the same in any
// order; the tokens' order is that of the keys below, whose difference to the largest one's is
// looked for digit by digit where a limit falls.
#include "rows.cuh"

namespace pv {
namespace {

constexpr int kSThreads = 512, kSWarps = kSThreads / 32;
constexpr int kBins = 2048;
using u64 = unsigned long long;

struct SampleShared {
    u64 bins[kBins], all[kBins];  // this CTA's, the cluster's
    u64 warp[kSWarps], cta[kMostCluster], found_before, found_weight;
    uint32_t found, key[kSWarps], ctakey[kMostCluster];
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

struct SampleArgs {
    SampleJob j;
    int ctas;  // of a row
};

struct Row {
    const SampleArgs &a;
    SampleShared &sh;
    int64_t t;
    int lane, warp;
    uint32_t rank, ctas;
    const char *base;  // the 16-byte boundary at or before the row
    int off, end;      // the row's tokens are off .. end - 1 from there
    int begin, last;   // tiles of this warp
    float m;
    const uint32_t *allowed;
    float big;         // the largest x

    __device__ __forceinline__ void meet() const {
        if (ctas > 1)
            clusters_meet();
        else
            __syncthreads();
    }
    // x of a lane's eight tokens of a tile, -infinity where there is none or it may not be chosen;
    // the first one's index.
    __device__ __forceinline__ int tokens(int tile, float (&x)[kWide]) const {
        const pvmvmd_rows &l = a.j.logits;
        const int at = tile * kTile + lane * kWide;
        Raw r;
        r.a = r.b = make_uint4(0, 0, 0, 0);
        if (two_bytes(l.type)) {
            if (at < end && at + kWide > off) r.a = *reinterpret_cast<const uint4 *>(base + (int64_t)at * 2);
        } else {
            if (at < end && at + 4 > off) r.a = *reinterpret_cast<const uint4 *>(base + (int64_t)at * 4);
            if (at + 4 < end && at + 8 > off) r.b = *reinterpret_cast<const uint4 *>(base + (int64_t)at * 4 + 16);
        }
        Two v2[kTwos];
        unpack(r, l.type, v2);
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[2 * i] = first(v2[i]), x[2 * i + 1] = second(v2[i]);
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
            float v = __fmul_rn(x[e], m);
            const bool in = i0 + e >= 0 && i0 + e < V;
            if (l.channel_scale_dev && in) v = __fmul_rn(v, l.channel_scale_dev[i0 + e]);
            v = v > -INFINITY ? fminf(v, kFltMax) : -INFINITY;  // (NaN is not)
            x[e] = in && (ok >> e & 1) ? v : -INFINITY;
        }
        return i0;
    }

    // f(x, index) for every token of this warp's tiles that may be chosen
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
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
            if (threadIdx.x == 0) sh.ctakey[0] = k;
            clusters_meet();
            k = __reduce_max_sync(kFull, lane < (int)ctas ? peer_u32(&sh.ctakey[0], (uint32_t)lane) : 0u);
        }
        meet();
        return k;
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
            u64 mine[kMine], sum = 0;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int b = (int)threadIdx.x * kMine + i;
                mine[i] = 0;
                for (uint32_t c = 0; c < ctas; ++c) mine[i] += ctas > 1 ? peer_u64(&sh.bins[b], c) : sh.bins[b];
                sum += mine[i];
            }
            u64 pre = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 u = __shfl_up_sync(kFull, pre, o);
                if (lane >= o) pre += u;
            }
            if (lane == 31) sh.warp[warp] = pre;
            meet();  // (the bins have been read, too)
            u64 total = 0;
            pre -= sum;
            for (int k = 0; k < kSWarps; ++k) {
                if (k < warp) pre += sh.warp[k];
                total += sh.warp[k];
            }
            pre += before;
            if (pre < target && pre + sum >= target) {
#pragma unroll
                for (int i = 0; i < kMine; ++i) {
                    if (pre < target && pre + mine[i] >= target) {
                        sh.found = threadIdx.x * kMine + i;
                        sh.found_before = pre;
                        sh.found_weight = mine[i];
                    }
                    pre += mine[i];
                }
            }
            __syncthreads();
            if (sh.found == ~0u) {  // in the first digit alone
                before += total;
                __syncthreads();
                return false;
            }
            v |= sh.found << open;
            before = sh.found_before;
            at = sh.found_weight;
            __syncthreads();
        }
        return true;
    }
};

// floor(v f / 2^31), f < 2^31
__device__ __forceinline__ u64 part_of(u64 v, uint32_t f31) { return __umul64hi(v, (u64)f31 << 33); }

// floor(2^31 p) of a part in [0, 1]
__device__ __forceinline__ uint32_t part31(float p) {
    return p > 0.0f ? (uint32_t)__fmul_rn(fminf(p, 1.0f), 2147483648.0f) : 0u;
}

__global__ void __launch_bounds__(kSThreads, 2) k_sample(const __grid_constant__ SampleArgs a) {
    follow();
    __shared__ SampleShared sh;
    const SampleJob &j = a.j;
    cluster_begin((uint32_t)a.ctas);
    Row r{a, sh};
    r.t = blockIdx.x / a.ctas;
    r.lane = threadIdx.x % 32;
    r.warp = threadIdx.x / 32;
    r.ctas = (uint32_t)a.ctas;
    r.rank = blockIdx.x % (uint32_t)a.ctas;
    const int V = j.V;
    const char *row = static_cast<const char *>(row_of(j.logits, j.logits.type, r.t));
    const int size = two_bytes(j.logits.type) ? 2 : 4, before16 = (int)(reinterpret_cast<uintptr_t>(row) % 16);
    r.base = row - before16;
    r.off = before16 / size;
    r.end = r.off + V;
    const int tiles = (r.end + kTile - 1) / kTile, per = (tiles + a.ctas * kSWarps - 1) / (a.ctas * kSWarps);
    r.begin = min(tiles, ((int)r.rank * kSWarps + r.warp) * per);
    r.last = min(tiles, r.begin + per);
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

    uint32_t key = 0;
    r.each([&](float x, int) { key = max(key, key_of(x)); });
    cluster_begun(r.ctas);
    const uint32_t top = r.max_key(key);
    const bool writes = threadIdx.x == 0 && r.rank == 0;
    if (top <= kNoKey) {
        if (writes) {
            j.token[r.t] = -1;
            if (j.logprob) j.logprob[r.t] = -INFINITY;
        }
        return;
    }
    r.big = of_key(top);
    if (greedy) {  // the lowest index, as the largest of its complement
        uint32_t low = 0;
        r.each([&](float x, int i) {
            if (key_of(x) == top) low = max(low, ~(uint32_t)i);
        });
        low = ~r.max_key(low);
        if (writes) {
            j.token[r.t] = (int)low;
            if (j.logprob) j.logprob[r.t] = 0.0f;
        }
        return;
    }

    // What is kept: values below cut, and of those at it the tokens up to cut_index.
    uint32_t cut = ~0u, cut_index = ~0u;
    u64 ties = 0, at_cut = 0;  // how many of those at it are kept; how many there are
    const bool by_k = top_k >= 1 && top_k < V, by_p = top_p < 1.0f;
    u64 before, at;
    if (by_k && r.reach(32, (u64)top_k, [&](float x, int, uint32_t &v, u64 &w) {
            v = top - key_of(x);
            w = 1;
            return true;
        }, cut, before, at)) {
        ties = (u64)top_k - before;
        at_cut = at;
    } else {
        cut = ~0u;
    }
    if (by_p) {
        auto below = [&](float x, int, uint32_t &v, u64 &w) {
            v = top - key_of(x);
            w = weight(r.big, x);
            return v < cut;
        };
        // (what is below the cut, from a target that is not reached)
        uint32_t v;
        r.reach(32, ~0ull, below, v, before, at);
        const u64 each = weight(r.big, of_key(top - cut)), kept = before + (cut == ~0u ? 0 : ties * each);
        const u64 target = max(part_of(kept, part31(top_p)), 1ull);
        if (r.reach(32, target, below, v, before, at)) {
            const u64 one = weight(r.big, of_key(top - v));
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
        r.reach(24, ties, [&](float x, int i, uint32_t &v, u64 &w) {
            v = (uint32_t)i;
            w = 1;
            return top - key_of(x) == cut;
        }, index, b, w1);
        cut_index = index;
    }

    // Z, the choice, and the tile and token where it falls
    const u64 least = (u64)part31(min_p) << 9;
    auto kept_weight = [&](float x, int i) {
        const uint32_t v = top - key_of(x);
        const u64 w = weight(r.big, x);
        return (v < cut || (v == cut && (uint32_t)i <= cut_index)) && w >= least ? w : 0ull;
    };
    u64 sum = 0;
    r.each([&](float x, int i) { sum += kept_weight(x, i); });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
    if (r.lane == 0) sh.warp[r.warp] = sum;
    __syncthreads();
    u64 mine = 0, front = 0, Z = 0;  // of this CTA; of what is in front of this warp; of all
    for (int k = 0; k < kSWarps; ++k) {
        mine += sh.warp[k];
        if (k < r.warp) front += sh.warp[k];
    }
    if (r.ctas > 1) {
        if (threadIdx.x == 0) sh.cta[0] = mine;
        clusters_meet();
        for (uint32_t c = 0; c < r.ctas; ++c) {
            const u64 v = peer_u64(&sh.cta[0], c);
            if (c < r.rank) front += v;
            Z += v;
        }
        clusters_meet();  // nothing of a CTA's is read once it may have ended
    } else {
        Z = mine;
    }
    const u64 at_random = __umul64hi(Z, (u64)j.random[r.t] << 32);
    if (at_random < front || at_random >= front + sum) return;
    for (int k = r.begin; k < r.last; ++k) {
        float x[kWide];
        const int i0 = r.tokens(k, x);
        u64 w[kWide], all = 0;
#pragma unroll
        for (int e = 0; e < kWide; ++e) all += w[e] = x[e] > -INFINITY ? kept_weight(x[e], i0 + e) : 0ull;
        u64 pre = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 u = __shfl_up_sync(kFull, pre, o);
            if (r.lane >= o) pre += u;
        }
        const u64 tile = __shfl_sync(kFull, pre, 31);
        pre += front - all;
        if (at_random >= pre && at_random < pre + all) {
#pragma unroll
            for (int e = 0; e < kWide; ++e) {
                if (at_random >= pre && at_random < pre + w[e]) {
                    j.token[r.t] = i0 + e;
                    if (j.logprob) j.logprob[r.t] = -log1pf(__fdiv_rn((float)(Z - w[e]), (float)w[e]));
                }
                pre += w[e];
            }
        }
        front += tile;
        if (at_random < front) return;
    }
}

}  // namespace

cudaError_t launch_sample(const SampleJob &j, cudaStream_t s) {
    SampleArgs a{j, 1};
    while (a.ctas < kMostCluster && (int64_t)j.T * a.ctas * 2 <= 304 && j.V / a.ctas >= 8192) a.ctas *= 2;
    return launch_cluster(k_sample, dim3((unsigned)(j.T * a.ctas)), a.ctas, kSThreads, 0, s, a);
}

}  // namespace pv
