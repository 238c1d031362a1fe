// Rows of values as the client's other steps read and write them (pvmvmd_rows and
// pvmvmd_rows_out of include/pvmvmd.h), and the arithmetic that these steps are defined in.
//
// The types are known at run time: what a thread reads first goes into registers as it
// is (Raw), so that all of its loads are under way before the first value is needed, and a branch
// that is the same for the whole grid turns it into 32-bit numbers.
#pragma once

#include <algorithm>

#include "attention.cuh"
#include "steps.h"

namespace pv {

constexpr float kFltMax = 3.402823466e+38f;
constexpr int kWide = 8;  // values that a thread takes at a time

__host__ __device__ inline bool two_bytes(int type) { return type == PVMVMD_BF16 || type == PVMVMD_F16; }

// Eight values as they lie in memory.
struct Raw {
    uint4 a, b;  // b: of 32-bit types alone
};

__device__ __forceinline__ float half_bits(uint32_t v, bool bf) {  // a 16-bit value
    return bf ? __uint_as_float(v << 16) : __half2float(__ushort_as_half((unsigned short)v));
}
__device__ __forceinline__ void unpack2(uint32_t v, bool bf, float &x, float &y) {
    if (bf) {
        x = __uint_as_float(v << 16);
        y = __uint_as_float(v & 0xffff0000u);
    } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v));
        x = f.x;
        y = f.y;
    }
}
// The values of a type, times nothing yet.
__device__ __forceinline__ void unpack(const Raw &r, int type, float (&x)[kWide]) {
    if (two_bytes(type)) {
        const bool bf = type == PVMVMD_BF16;
        unpack2(r.a.x, bf, x[0], x[1]);
        unpack2(r.a.y, bf, x[2], x[3]);
        unpack2(r.a.z, bf, x[4], x[5]);
        unpack2(r.a.w, bf, x[6], x[7]);
        return;
    }
    const uint32_t w[kWide] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
    if (type == PVMVMD_F32) {
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[e] = __uint_as_float(w[e]);
    } else {
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[e] = to_f32<uint32_t>(w[e]);
    }
}

// Where a thread's values lie in a row: eight side by side (kVec: rows on 16-byte boundaries,
// D a multiple of 8), or eight that are `step` apart, so that a warp's are side by side.
template <bool kVec>
struct Place {
    int at, step, D;  // the first, the distance of the others (1 where kVec)
    __device__ __forceinline__ int index(int e) const { return kVec ? at + e : at + e * step; }
    __device__ __forceinline__ bool in(int e) const { return index(e) < D; }
};

template <bool kVec>
__device__ __forceinline__ Raw load_raw(const void *row, int type, const Place<kVec> &p) {
    Raw r;
    if (kVec) {
        r.a = r.b = make_uint4(0, 0, 0, 0);
        if (p.at < p.D) {
            if (two_bytes(type)) {
                r.a = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(row) + p.at);
            } else {
                const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const uint32_t *>(row) + p.at);
                r.a = q[0];
                r.b = q[1];
            }
        }
        return r;
    }
    uint32_t w[kWide];
    if (two_bytes(type)) {
        const uint16_t *q = static_cast<const uint16_t *>(row);
#pragma unroll
        for (int e = 0; e < kWide; ++e) w[e] = p.in(e) ? q[p.index(e)] : 0;
        r.a = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        r.b = make_uint4(0, 0, 0, 0);
    } else {
        const uint32_t *q = static_cast<const uint32_t *>(row);
#pragma unroll
        for (int e = 0; e < kWide; ++e) w[e] = p.in(e) ? q[p.index(e)] : 0;
        r.a = make_uint4(w[0], w[1], w[2], w[3]);
        r.b = make_uint4(w[4], w[5], w[6], w[7]);
    }
    return r;
}

// A row's address: rows may be one for all.
__device__ __forceinline__ const void *row_of(const pvmvmd_rows &r, int64_t t) {
    return static_cast<const char *>(r.data_dev) + t * r.token * (two_bytes(r.type) ? 2 : 4);
}
// scale token_scale[t]
__device__ __forceinline__ float row_scale(const pvmvmd_rows &r, int64_t t) {
    return r.token_scale_dev ? __fmul_rn(r.scale, r.token_scale_dev[t]) : r.scale;
}

// 32-bit values of one row for all tokens: channel scales, or a norm's weights of any type.
template <bool kVec>
__device__ __forceinline__ void load_f32(const float *v, const Place<kVec> &p, float (&x)[kWide]) {
    unpack(load_raw<kVec>(v, PVMVMD_F32, p), PVMVMD_F32, x);
}

// Raw values to numbers: (x c) channel_scale
template <bool kVec>
__device__ __forceinline__ void read(const Raw &raw, const pvmvmd_rows &r, float c, const Place<kVec> &p, float (&x)[kWide]) {
    unpack(raw, r.type, x);
#pragma unroll
    for (int e = 0; e < kWide; ++e) x[e] = __fmul_rn(x[e], c);
    if (r.channel_scale_dev) {
        float s[kWide];
        load_f32<kVec>(r.channel_scale_dev, p, s);
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[e] = __fmul_rn(x[e], s[e]);
    }
}

// The integer of a value that has been multiplied, as a field element.
__device__ __forceinline__ uint32_t field_of(float v, float limit) {
    v = fminf(fmaxf(v, -limit), limit);
    const int n = __float2int_rn(v);
    return n < 0 ? (uint32_t)n + kQ : (uint32_t)n;
}

// Eight values to a row: a floating type, or integers by m.
template <bool kVec>
__device__ __forceinline__ void write(const pvmvmd_rows_out &o, int64_t t, const Place<kVec> &p, const float (&z)[kWide],
                                      float m) {
    if (o.type == PVMVMD_BF16 || o.type == PVMVMD_F16) {
        uint16_t *row = static_cast<uint16_t *>(o.data_dev) + t * o.token;
        uint32_t w[kWide / 2];
#pragma unroll
        for (int e = 0; e < kWide / 2; ++e) {
            if (o.type == PVMVMD_BF16) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(z[2 * e], z[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t *>(&v);
            } else {
                const __half2 v = __floats2half2_rn(z[2 * e], z[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t *>(&v);
            }
        }
        if (kVec) {
            if (p.at < p.D) *reinterpret_cast<uint4 *>(row + p.at) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int e = 0; e < kWide; ++e)
                if (p.in(e)) row[p.index(e)] = (uint16_t)(e & 1 ? w[e / 2] >> 16 : w[e / 2]);
        }
        return;
    }
    uint32_t w[kWide];
    if (o.type == PVMVMD_F32) {
#pragma unroll
        for (int e = 0; e < kWide; ++e) w[e] = __float_as_uint(z[e]);
    } else {
        const float limit = (float)o.limit;
#pragma unroll
        for (int e = 0; e < kWide; ++e) {
            const float v = __fmul_rn(z[e], m);
            w[e] = v == v ? field_of(v, limit) : 0u;
        }
    }
    uint32_t *row = static_cast<uint32_t *>(o.data_dev) + t * o.token;
    if (kVec) {
        if (p.at < p.D) {
            uint4 *q = reinterpret_cast<uint4 *>(row + p.at);
            q[0] = make_uint4(w[0], w[1], w[2], w[3]);
            q[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kWide; ++e)
            if (p.in(e)) row[p.index(e)] = w[e];
    }
}

// What a row's integers are multiplied by, from the largest |z| (as bits), and its step.  A row that is not finite:
// m = 0 gives zeros for what is finite, NaN (zeros) for what is not.
__device__ __forceinline__ float dynamic_scale(const pvmvmd_rows_out &o, uint32_t big, float &step) {
    if (big >= 0x7f800000u) {
        step = __uint_as_float(0x7fffffffu);
        return 0.0f;
    }
    const float a = __uint_as_float(big), limit = (float)o.limit;
    step = __fdiv_rn(a, limit);
    return fminf(__fdiv_rn(limit, a), kFltMax);
}

// ---------------------------------------------------------------- powers of two
// 2^-f, |f| <= 1/2: the polynomial of degree 5 that is 1 at 0 and whose largest relative
// error is least (2^-23.4; found by weighted least squares), products and sums rounded
// one by one (2^-22.3 in all).
__device__ __forceinline__ float exp_poly(float f) {
    float p = __fadd_rn(__fmul_rn(f, -0.00132647157f), 0.00967151299f);
    p = __fadd_rn(__fmul_rn(p, f), -0.0555073395f);
    p = __fadd_rn(__fmul_rn(p, f), 0.240222424f);
    p = __fadd_rn(__fmul_rn(p, f), -0.693147004f);
    return __fadd_rn(__fmul_rn(p, f), 1.0f);
}
// d = n + f, n the nearest whole number (adding 1.5 2^23 rounds to it), |d| <= 2^22
__device__ __forceinline__ float split(float d, int &n) {
    const float t = __fadd_rn(d, 12582912.0f);
    n = __float_as_int(t) - 0x4b400000;
    return __fsub_rn(d, __fsub_rn(t, 12582912.0f));
}
// 1 + 2^-d
__device__ __forceinline__ float one_plus_exp(float d) {
    int n;
    const float p = exp_poly(split(fminf(fmaxf(d, -128.0f), 125.0f), n));
    return __fadd_rn(1.0f, __int_as_float(__float_as_int(p) - (n << 23)));
}

// ---------------------------------------------------------------- sums in pairs
// h + l, |l| about 2^-24 |h|: sums and squares to about 2^-45 of the sum of their terms'
// sizes (Dekker, Numer. Math. 1971; Knuth, TAOCP vol. 2, 4.2.2).
struct Pair {
    float h, l;
};
__device__ __forceinline__ void add_term(Pair &s, float x, float low) {
    const float t = __fadd_rn(s.h, x), b = __fsub_rn(t, s.h);
    const float e = __fadd_rn(__fsub_rn(s.h, __fsub_rn(t, b)), __fsub_rn(x, b));
    s.h = t;
    s.l = __fadd_rn(s.l, __fadd_rn(e, low));
}
__device__ __forceinline__ void add_square(Pair &s, float x) {
    const float p = __fmul_rn(x, x);
    add_term(s, p, __fmaf_rn(x, x, -p));
}
// s / n for a whole number n < 2^24
__device__ __forceinline__ Pair mean_of(Pair s, float n) {
    const float h = __fadd_rn(s.h, s.l), l = __fadd_rn(__fsub_rn(s.h, h), s.l);
    const float q = __fdiv_rn(h, n);
    return Pair{q, __fdiv_rn(__fadd_rn(__fmaf_rn(-q, n, h), l), n)};
}
// 1 / sqrt(a + eps), rounded once: the approximation y of a's upper part, corrected by
// what 1 - a y^2 is in twice the bits.
__device__ __forceinline__ float inverse_root(Pair a, float eps) {
    Pair s{a.h, a.l};
    add_term(s, eps, 0.0f);
    const float h = __fadd_rn(s.h, s.l), l = __fadd_rn(__fsub_rn(s.h, h), s.l);
    const float y = rsqrtf(h), t = __fmul_rn(y, y), te = __fmaf_rn(y, y, -t);
    const float r = -__fmaf_rn(l, t, __fmaf_rn(h, te, __fmaf_rn(h, t, -1.0f)));
    return __fmaf_rn(y, __fmul_rn(r, __fmaf_rn(0.375f, r, 0.5f)), y);
}

// ---------------------------------------------------------------- across a row's threads
// A row's threads: the lanes of a warp, the warps of a CTA, the CTAs of a cluster.  Every
// exchange has a place of its own in shared memory, so that none waits for the reads
// of the one before, and every thread gets the same result.
constexpr int kMostCluster = 8, kMostWarps = 32, kExchanges = 5;
struct RowShared {
    Pair warp[kExchanges][kMostWarps];
    Pair cta[kExchanges][kMostCluster];
};
struct RowThreads {
    RowShared *sh;
    int warps;             // 1: a warp by itself, with others' rows beside it
    int lane, warp, used;  // used: exchanges so far
    uint32_t ctas, rank;
};

__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cta_count() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
// At a kernel's start and before its first store to a peer: all of the cluster's CTAs run.
__device__ __forceinline__ void cluster_begin(uint32_t ctas) {
    if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_begun(uint32_t ctas) {
    if (ctas > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ void clusters_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A value of 8 bytes to shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ void store_peer(const void *p, uint32_t rank, Pair v) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.h), "f"(v.l) : "memory");
}

// op(a, b) is the same for (b, a); neutral: op(a, neutral) = a.
template <typename Op>
__device__ __forceinline__ Pair reduce_lanes(Pair v, int from, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o <= from)
            v = op(v, Pair{__shfl_xor_sync(kFull, v.h, o), __shfl_xor_sync(kFull, v.l, o)});
    return v;
}
template <typename Op>
__device__ __forceinline__ Pair reduce_row(RowThreads &r, Pair v, Pair neutral, Op op) {
    v = reduce_lanes(v, 16, op);
    if (r.warps == 1) return v;
    Pair *mine = r.sh->warp[r.used];
    if (r.lane == 0) mine[r.warp] = v;
    __syncthreads();
    v = r.lane < r.warps ? mine[r.lane] : neutral;
    v = reduce_lanes(v, 16, op);
    if (r.ctas > 1) {
        Pair *all = r.sh->cta[r.used];
        if (r.used == 0) cluster_begun(r.ctas);
        if (r.warp == 0 && r.lane < (int)r.ctas) store_peer(&all[r.rank], (uint32_t)r.lane, v);
        clusters_meet();
        v = r.lane < (int)r.ctas ? all[r.lane] : neutral;
        v = reduce_lanes(v, kMostCluster / 2, op);
        v = Pair{__shfl_sync(kFull, v.h, 0), __shfl_sync(kFull, v.l, 0)};
    }
    ++r.used;
    return v;
}
__device__ __forceinline__ Pair row_sum(RowThreads &r, Pair v) {
    return reduce_row(r, v, Pair{0.0f, 0.0f}, [](Pair a, Pair b) {
        // symmetric, so that all lanes hold the same bits
        const float t = __fadd_rn(a.h, b.h), bb = __fsub_rn(t, a.h);
        const float e = __fadd_rn(__fsub_rn(a.h, __fsub_rn(t, bb)), __fsub_rn(b.h, bb));
        return Pair{t, __fadd_rn(__fadd_rn(a.l, b.l), e)};
    });
}
__device__ __forceinline__ uint32_t row_max(RowThreads &r, uint32_t v) {
    v = __reduce_max_sync(kFull, v);
    if (r.warps == 1) return v;
    const Pair m = reduce_row(r, Pair{__uint_as_float(v), 0.0f}, Pair{0.0f, 0.0f}, [](Pair a, Pair b) {
        return Pair{__uint_as_float(max(__float_as_uint(a.h), __float_as_uint(b.h))), 0.0f};
    });
    return __float_as_uint(m.h);
}

// A row's threads never exchanged anything: the wait that goes with cluster_begin.
__device__ __forceinline__ void row_end(const RowThreads &r) {
    if (r.used == 0) cluster_begun(r.ctas);
}

// How rows are dealt to threads: rows of up to 1024 values to a warp each, others to a CTA
// or to a cluster of them; a thread takes `chunks` times eight values.
constexpr int kRowThreadsMost = 512, kWarpRows = 8;
struct RowDeal {
    int threads;  // of a CTA
    int rows;     // of a CTA: one a warp, or one
    int ctas;     // of a row
    int chunks;   // 1, 2 or 4
};
inline RowDeal deal_rows(int T, int D) {
    const int units = (D + kWide - 1) / kWide;
    RowDeal d{32, 1, 1, 1};
    if (units <= 4 * 32) {
        while (units > 32 * d.chunks) d.chunks *= 2;
        d.rows = std::max(1, std::min(kWarpRows, T / 152));
        d.threads = 32 * d.rows;
        return d;
    }
    d.chunks = T >= 152 ? 2 : 1;
    while (units > kRowThreadsMost * d.chunks * d.ctas && d.ctas < kMostCluster) d.ctas *= 2;
    while (units > kRowThreadsMost * d.chunks * d.ctas) d.chunks *= 2;
    const int each = (units + d.ctas * d.chunks - 1) / (d.ctas * d.chunks);
    d.threads = (each + 31) / 32 * 32;
    return d;
}
// The place of a thread's chunk c among the values of its row.
template <bool kVec>
__device__ __forceinline__ Place<kVec> place_of(const RowThreads &r, int threads, int chunk, int chunks, int D) {
    // of a CTA's part, chunks one after the other, threads side by side
    const int width = r.warps == 1 ? 32 : threads, tid = r.warps == 1 ? r.lane : r.warp * 32 + r.lane;
    const int first = ((int)r.rank * chunks + chunk) * width * kWide;
    return kVec ? Place<kVec>{first + tid * kWide, 1, D} : Place<kVec>{first + tid, width, D};
}
__device__ __forceinline__ RowThreads row_threads(RowShared *sh, const RowDeal &d) {
    RowThreads r;
    r.sh = sh;
    r.lane = threadIdx.x % 32;
    r.warp = threadIdx.x / 32;
    r.warps = d.rows > 1 || d.threads == 32 ? 1 : d.threads / 32;
    r.ctas = (uint32_t)d.ctas;
    r.rank = d.ctas > 1 ? cta_rank() : 0;
    r.used = 0;
    return r;
}

// Whether a row's values can be taken 16 bytes at a time.
inline bool whole16(const void *p, int64_t stride, int type) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (two_bytes(type) ? 2 : 4) % 16 == 0;
}
inline bool whole16(const pvmvmd_rows &r) {
    return whole16(r.data_dev, r.token, r.type) && whole16(r.channel_scale_dev, 0, PVMVMD_F32);
}
inline bool whole16(const pvmvmd_rows_out &o) { return whole16(o.data_dev, o.token, o.type); }

}  // namespace pv
