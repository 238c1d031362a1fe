// Rows of values as the client's other steps read and write them (pvmvmd_rows and
// pvmvmd_rows_out of include/pvmvmd.h), and the arithmetic that these steps are defined in.
//
// What a thread reads first goes into registers as it is (Raw), so that all of its loads are under way
// before the first value is needed, and then becomes 32-bit numbers, by a branch that is the same for
// the whole grid where the kernel is compiled for any type.
#pragma once

#include <algorithm>
#include <climits>

#include "attention.cuh"
#include "steps.h"

namespace pv {

constexpr float kFltMax = 3.402823466e+38f;
constexpr int kWide = 8;  // values that a thread takes at a time
constexpr int kTwos = kWide / 2;
constexpr int kSms = 152;  // of the GPU that the library is compiled for; the rules that use it were measured there

__host__ __device__ inline bool two_bytes(int type) { return type == PVMVMD_BF16 || type == PVMVMD_F16; }

// What a kernel is compiled for: values of one type, or (0) of any.
constexpr int kAny = 0, kBf16 = PVMVMD_BF16, kF16 = PVMVMD_F16, kF32 = PVMVMD_F32, kField = PVMVMD_FIELD;
template <int k>
__device__ __forceinline__ int known(int type) {
    return k == kAny ? type : k;
}

// ---------------------------------------------------------------- two numbers at a time
// Products and sums of pairs by one instruction, each rounded by itself as if alone.  They are kept as the
// 64 bits that the instruction takes: as two of 32 they would be moved together every time.
struct Two {
    unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ Two two(uint32_t a, uint32_t b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ Two both(float v) { return two(v, v); }
__device__ __forceinline__ float first(Two x) { return __uint_as_float((uint32_t)x.v); }
__device__ __forceinline__ float second(Two x) { return __uint_as_float((uint32_t)(x.v >> 32)); }
__device__ __forceinline__ Two add2(Two x, Two y) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(x.v), "l"(y.v));
    return r;
}
__device__ __forceinline__ Two sub2(Two x, Two y) {
    Two r;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(x.v), "l"(y.v));
    return r;
}
__device__ __forceinline__ Two fma2(Two x, Two y, Two z) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(x.v), "l"(y.v), "l"(z.v));
    return r;
}
__device__ __forceinline__ Two minus2(Two x) { return Two{x.v ^ 0x8000000080000000ull}; }
// A product alone.  (mul.rn.f32x2 and an add.rn.f32x2 after it are joined by the assembler of CUDA 13.0 to one
// rounding, also under -fmad=false; so are a product plus a constant -0 and a sum times a constant 1.  With a -0
// that only the running kernel knows there is nothing to join.)
static __constant__ float s_minus_zero = -0.0f;
__device__ __forceinline__ Two mul2(Two x, Two y) { return fma2(x, y, both(s_minus_zero)); }

// ---------------------------------------------------------------- reading
// Eight values as they lie in memory.
struct Raw {
    uint4 a, b;  // b: of 32-bit types alone
};

__device__ __forceinline__ Two half2_of(uint32_t v) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v));
    return two(f.x, f.y);
}
__device__ __forceinline__ Two bfloat2_of(uint32_t v) { return two(v << 16, v & 0xffff0000u); }
// The values of a type, times nothing yet.
__device__ __forceinline__ void unpack(const Raw &r, int type, Two (&x)[kTwos]) {
    const uint32_t h[kTwos] = {r.a.x, r.a.y, r.a.z, r.a.w};
    if (type == PVMVMD_BF16) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = bfloat2_of(h[i]);
        return;
    }
    if (type == PVMVMD_F16) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = half2_of(h[i]);
        return;
    }
    const uint32_t w[kWide] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < kTwos; ++i)
        x[i] = type == PVMVMD_F32 ? two(w[2 * i], w[2 * i + 1])
                                  : two(to_f32<uint32_t>(w[2 * i]), to_f32<uint32_t>(w[2 * i + 1]));
}

// Where a thread's values lie in a row: a warp takes 256 at a time, a lane eight of them, which are side by
// side (kVec: rows on 16-byte boundaries, D a multiple of 8, so that all are in the row or none), or 32
// apart, so that the warp's are side by side.
constexpr int kTile = 32 * kWide;
template <bool kVec>
struct Place {
    int at, D;
    __device__ __forceinline__ bool any() const { return at < D; }
    __device__ __forceinline__ int index(int e) const { return kVec ? at + e : at + e * 32; }
    __device__ __forceinline__ bool in(int e) const { return kVec ? at < D : index(e) < D; }
    // of a thread's chunk c, counted from its first
    __device__ __forceinline__ Place chunk(int c) const { return Place{at + c * kTile, D}; }
};

template <bool kVec>
__device__ __forceinline__ Raw load_raw(const void *row, int type, const Place<kVec> &p) {
    Raw r;
    if (kVec) {
        r.a = r.b = make_uint4(0, 0, 0, 0);
        if (p.any()) {
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
__device__ __forceinline__ const void *row_of(const pvmvmd_rows &r, int type, int64_t t) {
    return static_cast<const char *>(r.data_dev) + t * r.token * (two_bytes(type) ? 2 : 4);
}
// scale token_scale[t]
__device__ __forceinline__ float row_scale(const pvmvmd_rows &r, int64_t t) {
    return r.token_scale_dev ? __fmul_rn(r.scale, r.token_scale_dev[t]) : r.scale;
}

// Raw values to numbers: (x c) channel_scale
template <bool kVec>
__device__ __forceinline__ void read(const Raw &raw, const pvmvmd_rows &r, int type, float c, const Place<kVec> &p,
                                     Two (&x)[kTwos]) {
    unpack(raw, type, x);
#pragma unroll
    for (int i = 0; i < kTwos; ++i) x[i] = mul2(x[i], both(c));
    if (r.channel_scale_dev) {
        Two s[kTwos];
        unpack(load_raw<kVec>(r.channel_scale_dev, PVMVMD_F32, p), PVMVMD_F32, s);
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = mul2(x[i], s[i]);
    }
}
// Zeros in the place of what lies outside the row.
template <bool kVec>
__device__ __forceinline__ void outside_zero(const Place<kVec> &p, Two (&x)[kTwos]) {
    if (kVec && p.any()) return;
#pragma unroll
    for (int i = 0; i < kTwos; ++i)
        x[i] = two(p.in(2 * i) ? first(x[i]) : 0.0f, p.in(2 * i + 1) ? second(x[i]) : 0.0f);
}

// ---------------------------------------------------------------- writing
// A number of up to kMostLimit rounded to a whole one, halves to even, as a field element: adding
// 1.5 2^23 leaves the whole number in the sum's lower bits; of n and n + q, read without signs, the
// smaller one is canonical.
__device__ __forceinline__ uint32_t field_of(float v) {
    const uint32_t b = __float_as_uint(__fadd_rn(v, 12582912.0f));
    return min(b - 0x4b400000u, b + (kQ - 0x4b400000u));
}

// What becomes of a row's values: by_row: m is the row's own, so that every |z m| is below limit + 1/2,
// or 0 where the row is not finite.
struct Step {
    float m;
    bool by_row;
};

// Eight values to a row: a floating type, or integers.
template <bool kVec>
__device__ __forceinline__ void write(const pvmvmd_rows_out &o, int type, int64_t t, const Place<kVec> &p,
                                      const Two (&z)[kTwos], Step s) {
    if (two_bytes(type)) {
        uint16_t *row = static_cast<uint16_t *>(o.data_dev) + t * o.token;
        uint32_t w[kTwos];
        if (type == PVMVMD_BF16) {
#pragma unroll
            for (int i = 0; i < kTwos; ++i) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(first(z[i]), second(z[i]));
                w[i] = *reinterpret_cast<const uint32_t *>(&v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kTwos; ++i) {
                const __half2 v = __floats2half2_rn(first(z[i]), second(z[i]));
                w[i] = *reinterpret_cast<const uint32_t *>(&v);
            }
        }
        if (kVec) {
            if (p.any()) *reinterpret_cast<uint4 *>(row + p.at) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int e = 0; e < kWide; ++e)
                if (p.in(e)) row[p.index(e)] = (uint16_t)(e & 1 ? w[e / 2] >> 16 : w[e / 2]);
        }
        return;
    }
    uint32_t w[kWide];
    if (type == PVMVMD_F32) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) {
            w[2 * i] = __float_as_uint(first(z[i]));
            w[2 * i + 1] = __float_as_uint(second(z[i]));
        }
    } else if (s.by_row && s.m != 0.0f) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) {
            const Two v = mul2(z[i], both(s.m));
            w[2 * i] = field_of(first(v));
            w[2 * i + 1] = field_of(second(v));
        }
    } else {
        const float limit = (float)o.limit;
#pragma unroll
        for (int i = 0; i < kTwos; ++i) {
            Two v = mul2(z[i], both(s.m));
            w[2 * i] = first(v) == first(v) ? field_of(fminf(fmaxf(first(v), -limit), limit)) : 0u;
            w[2 * i + 1] = second(v) == second(v) ? field_of(fminf(fmaxf(second(v), -limit), limit)) : 0u;
        }
    }
    uint32_t *row = static_cast<uint32_t *>(o.data_dev) + t * o.token;
    if (kVec) {
        if (p.any()) {
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

// The larger of a and |b|; NaN if one is.
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
// What a row's integers are multiplied by, from its largest |z|, and its step.  A row that is not finite:
// m = 0 gives zeros for what is finite, NaN (zeros) for what is not.
__device__ __forceinline__ Step step_of(const pvmvmd_rows_out &o, float big) {
    if (!(big <= kFltMax)) return Step{0.0f, true};
    return Step{fminf(__fdiv_rn((float)o.limit, big), kFltMax), true};
}
__device__ __forceinline__ void write_step(const pvmvmd_rows_out &o, int64_t t, float big) {
    o.token_scale_dev[t] = big <= kFltMax ? __fdiv_rn(big, (float)o.limit) : __uint_as_float(0x7fffffffu);
}

// ---------------------------------------------------------------- powers of two
// 2^-f, |f| <= 1/2: the polynomial of degree 5 that is 1 at 0 and whose largest relative
// error is least (2^-23.4; found by weighted least squares), products and sums rounded
// one by one (2^-22.3 in all).  gain: a power of two that the result is multiplied by (which
// rounds nothing).
__device__ __forceinline__ Two exp_poly(Two f, float gain = 1.0f) {
    Two p = add2(mul2(f, both(-0.00132647157f * gain)), both(0.00967151299f * gain));
    p = add2(mul2(p, f), both(-0.0555073395f * gain));
    p = add2(mul2(p, f), both(0.240222424f * gain));
    p = add2(mul2(p, f), both(-0.693147004f * gain));
    return add2(mul2(p, f), both(gain));
}
// d = n + f, n the nearest whole number (adding 1.5 2^23 rounds to it), |d| <= 2^22.  Returns f; n + 0x4b400000
// is what the bits of `sum` are.
__device__ __forceinline__ Two split(Two d, Two &sum) {
    sum = add2(d, both(12582912.0f));
    return sub2(d, sub2(sum, both(12582912.0f)));
}
// 2^-d for |d| < 127.  (23 bits up, nothing is left of 0x4b400000.)
__device__ __forceinline__ Two power_near(Two d) {
    Two n;
    const Two p = exp_poly(split(d, n));
    return two((uint32_t)p.v - ((uint32_t)n.v << 23), (uint32_t)(p.v >> 32) - ((uint32_t)(n.v >> 32) << 23));
}
// 2^-d for d cut to [-128, 125], infinity at -128.
__device__ __forceinline__ Two power(Two d) {
    return power_near(two(fminf(fmaxf(first(d), -128.0f), 125.0f), fminf(fmaxf(second(d), -128.0f), 125.0f)));
}

// ---------------------------------------------------------------- sums in pairs
// h + l, |l| about 2^-24 |h|: sums and squares to about 2^-45 of the sum of their terms'
// sizes (Dekker, Numer. Math. 1971; Knuth, TAOCP vol. 2, 4.2.2).  At worst, of 16 terms in a row l takes an error of
// 2^-24 of the sum with each, and as many of its own of 2^-24 of what it has, in all (1 + 2 + .. + 16 + 48) 2^-48; a
// warp's sum below adds 32 of 2^-25 in 2^21 or more, that of 16 warps half of it and that of 8 CTAs a quarter: below 2^-39.
// What falls below 2^-149 is lost: 2^-150 and 2^-149 of each term, and 2^-149 of each lane's sum.
struct Pair {
    float h, l;
};
inline Pair inverse_of(int n) {
    const float h = (float)(1.0 / n);
    return Pair{h, (float)(1.0 / n - h)};
}
struct Pairs {  // two of them
    Two h, l;
};
__device__ __forceinline__ void add_terms(Pairs &s, Two x) {
    const Two t = add2(s.h, x), b = sub2(t, s.h);
    s.l = add2(s.l, add2(sub2(s.h, sub2(t, b)), sub2(x, b)));
    s.h = t;
}
__device__ __forceinline__ void add_squares(Pairs &s, Two x) {
    const Two p = mul2(x, x), low = fma2(x, x, minus2(p)), t = add2(s.h, p), b = sub2(t, s.h);
    s.l = add2(s.l, add2(add2(sub2(s.h, sub2(t, b)), sub2(p, b)), low));
    s.h = t;
}
__device__ __forceinline__ Pair join(Pair a, Pair b) {  // the same for (b, a)
    const float t = __fadd_rn(a.h, b.h), bb = __fsub_rn(t, a.h);
    const float e = __fadd_rn(__fsub_rn(a.h, __fsub_rn(t, bb)), __fsub_rn(b.h, bb));
    return Pair{t, __fadd_rn(__fadd_rn(a.l, b.l), e)};
}
__device__ __forceinline__ Pair join(const Pairs &s) { return join(Pair{first(s.h), first(s.l)}, Pair{second(s.h), second(s.l)}); }
// s / n rounded once, by the rounded inverse of n.  The quotient's rest is exact (18 bits), and so is its n-th part
// (Markstein, IBM J. Res. Dev. 34, 1990) where s / n is the middle of two numbers, as rows of few different values often
// have it: the even one is taken.
__device__ __forceinline__ float rounded_mean(Pair s, float n, float inverse) {
    const float h = __fadd_rn(s.h, s.l), l = __fadd_rn(__fsub_rn(s.h, h), s.l), q = __fmul_rn(h, inverse);
    const float rest = __fadd_rn(__fmaf_rn(-q, n, h), l), part = __fmul_rn(rest, inverse);
    return __fadd_rn(q, __fmaf_rn(__fmaf_rn(-part, n, rest), inverse, part));
}
// s (1 / n), the latter a pair of the host's
__device__ __forceinline__ Pair mean_of(Pair s, Pair inverse) {
    const float h = __fadd_rn(s.h, s.l), l = __fadd_rn(__fsub_rn(s.h, h), s.l), p = __fmul_rn(h, inverse.h);
    return Pair{p, __fmaf_rn(l, inverse.h, __fmaf_rn(h, inverse.l, __fmaf_rn(h, inverse.h, -p)))};
}
// 1 / sqrt(a + eps), rounded once: the approximation y of a's upper part, corrected by
// what 1 - a y^2 is in twice the bits.  Of sums far from 1, whose y^2 or its lower 24 bits 32-bit numbers do not
// hold, it is taken of the sum times a power of four, which comes off the root exactly.  (Of all sums: 8192 x 8192 155.8 us,
// 154.3 so.)
__device__ __forceinline__ float inverse_root(Pair a, float eps) {
    const Pair s = join(a, Pair{eps, 0.0f});
    float h = __fadd_rn(s.h, s.l), l = __fadd_rn(__fsub_rn(s.h, h), s.l), back = 1.0f;
    if (!(h >= 0x1p-100f && h <= 0x1p100f)) {
        const bool below1 = h < 1.0f;
        const float gain = below1 ? 0x1p64f : 0x1p-64f;
        h = __fmul_rn(h, gain);
        l = __fmul_rn(l, gain);
        back = below1 ? 0x1p32f : 0x1p-32f;
    }
    const float y = rsqrtf(h), t = __fmul_rn(y, y), te = __fmaf_rn(y, y, -t), root = __fmul_rn(y, back);
    const float r = -__fmaf_rn(l, t, __fmaf_rn(h, te, __fmaf_rn(h, t, -1.0f)));
    return __fmaf_rn(root, __fmul_rn(r, __fmaf_rn(0.375f, r, 0.5f)), root);
}

// ---------------------------------------------------------------- across a row's threads
// How rows are dealt to threads: rows of up to 512 values to a warp each, others to a CTA
// or to a cluster of them; a thread takes `chunks` times eight values.
constexpr int kRowThreadsMost = 512, kWarpRows = 8, kMostCluster = 8, kMostWarps = kRowThreadsMost / 32;
struct RowDeal {
    int threads;   // of a CTA
    int rows;      // of a CTA: one a warp, or one
    int log_ctas;  // CTAs of a row: 2^log_ctas
    int chunks;    // 1, 2 or 4
    bool joint;    // the CTAs of a row are a cluster
};

// A row's threads: the lanes of a warp, the warps of a CTA, the CTAs of a cluster.  Every
// exchange has a place of its own in shared memory, so that none waits for the reads
// of the one before.
constexpr int kPlaces = 5;
struct RowShared {
    Pair warp[kPlaces][kMostWarps];
    Pair cta[kPlaces][kMostCluster];
};
struct RowThreads {
    RowShared *sh;
    int warps;              // 1: a warp by itself, with others' rows beside it
    int lane, warp, place;  // place: of the next exchange
    uint32_t ctas, rank;
    int64_t t;              // the row
};

// At a kernel's start, and before its first store to a peer: all of the cluster's CTAs run.
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

// The sum over a warp's lanes, the same in all: as whole numbers in units of 2^-46 of the power of two
// above the largest, in two parts that the warp adds in one instruction each.  (Five steps
// of shuffles and sums of pairs take three times the instructions.)  NaN where a value is not
// finite.
__device__ __forceinline__ Pair lanes_sum(Pair v) {
    const float h = __fadd_rn(v.h, v.l), l = __fadd_rn(__fsub_rn(v.h, h), v.l);
    const uint32_t most = __reduce_max_sync(kFull, __float_as_uint(h) & 0x7fffffffu);
    if (most >= 0x7f800000u) return Pair{__uint_as_float(0x7fffffffu), 0.0f};
    const uint32_t e = max(most >> 23, 24u);
    const float up = __uint_as_float((275u - e) << 23), down = __uint_as_float((e - 21u) << 23);  // 2^(148-e), its inverse
    const float a = __fmul_rn(h, up);                      // |a| < 2^22
    const float whole = __fadd_rn(a, 12582912.0f);         // 1.5 2^23: rounds to whole numbers
    const float rest = __fmaf_rn(l, up, __fsub_rn(a, __fsub_rn(whole, 12582912.0f)));  // |rest| < 1
    const int n = __reduce_add_sync(kFull, __float_as_int(whole) - 0x4b400000);
    const int m = __reduce_add_sync(kFull, __float2int_rn(__fmul_rn(rest, 16777216.0f)));
    // n + 2^-24 m: n may have more than 24 bits
    const float nh = __int2float_rn(n), nl = __int2float_rn(n - (int)nh);
    return Pair{__fmul_rn(nh, down), __fmul_rn(__fmaf_rn(__int2float_rn(m), 5.9604644775390625e-8f, nl), down)};
}
// Before the first store to a peer, or at the end where there is none.
__device__ __forceinline__ void row_begun(const RowThreads &r) {
    if (r.place == 0) cluster_begun(r.ctas);
}
__device__ __forceinline__ Pair row_sum(RowThreads &r, Pair v) {
    v = lanes_sum(v);
    if (r.warps == 1) return v;
    Pair *mine = r.sh->warp[r.place];
    if (r.lane == 0) mine[r.warp] = v;
    __syncthreads();
    v = lanes_sum(r.lane < r.warps ? mine[r.lane] : Pair{0.0f, 0.0f});
    if (r.ctas > 1) {
        Pair *all = r.sh->cta[r.place];
        row_begun(r);
        if (r.warp == 0 && r.lane < (int)r.ctas) store_peer(&all[r.rank], (uint32_t)r.lane, v);
        clusters_meet();
        v = lanes_sum(r.lane < (int)r.ctas ? all[r.lane] : Pair{0.0f, 0.0f});
    }
    ++r.place;
    return v;
}
// The largest of values that are not below 0; NaN if one is (whose bits are above all others').
__device__ __forceinline__ float row_max(RowThreads &r, float value) {
    uint32_t v = __reduce_max_sync(kFull, __float_as_uint(value));
    if (r.warps > 1) {
        Pair *mine = r.sh->warp[r.place];
        if (r.lane == 0) mine[r.warp].h = __uint_as_float(v);
        __syncthreads();
        v = __reduce_max_sync(kFull, r.lane < r.warps ? __float_as_uint(mine[r.lane].h) : 0u);
        if (r.ctas > 1) {
            Pair *all = r.sh->cta[r.place];
            row_begun(r);
            if (r.warp == 0 && r.lane < (int)r.ctas) store_peer(&all[r.rank], (uint32_t)r.lane, Pair{__uint_as_float(v), 0.0f});
            clusters_meet();
            v = __reduce_max_sync(kFull, r.lane < (int)r.ctas ? __float_as_uint(all[r.lane].h) : 0u);
        }
        ++r.place;
    }
    return __uint_as_float(v);
}

// joint: the row's CTAs have something to tell one another.
inline RowDeal deal_rows(int T, int D, bool joint) {
    const int tiles = (D + kTile - 1) / kTile, most = kRowThreadsMost / 32;
    RowDeal d{32, 1, 0, 1, joint};
    if (tiles <= 2) {
        d.chunks = tiles;
        d.rows = std::max(1, std::min(kWarpRows, T / kSms));
        d.threads = 32 * d.rows;
        return d;
    }
    // Few rows: as many threads as can be, each waiting for little.  Of many, two chunks a thread let two rows' CTAs run
    // on an SM.  (Norms to integers with a step a row, one chunk and two.  8 rows: of 4096 3.7 and 3.2 us, of 8192 3.8 and 4.4,
    // of 16384 4.0 and 5.5; 64: 4.0 and 3.4, 4.4 and 4.5, 6.1 and 5.7; 128: 4.4 and 3.4, 5.9 and 4.7, 12.1 and 9.5; 2048: 31
    // and 20, 79 and 40, 158 and 100.)
    d.chunks = T > 100 ? 2 : 1;
    // Few rows: CTAs of about four warps, as many as two an SM, since each waits for its own loads alone (one row of 8192
    // between two norms 5.2 us with a cluster of 2, 4.1 with one of 8; 64 rows 5.5 and, with 4, 5.1).
    if (d.chunks == 1)
        while (tiles > 4 << d.log_ctas && d.log_ctas < 3 && (T << (d.log_ctas + 1)) <= 2 * kSms) ++d.log_ctas;
    // CTAs of 8 warps where they need not wait for one another, else as few as there can be
    while (tiles > (joint ? most : 8) * d.chunks << d.log_ctas && (d.log_ctas < 3 || !joint)) ++d.log_ctas;
    while (tiles > most * d.chunks << d.log_ctas) d.chunks *= 2;
    d.threads = 32 * ((tiles + (d.chunks << d.log_ctas) - 1) / (d.chunks << d.log_ctas));
    return d;
}
// (No CTAs, which no launch takes, where there are more than a grid has.)
inline dim3 grid_of(const RowDeal &d, int T) {
    const int64_t n = (((int64_t)T + d.rows - 1) / d.rows) << d.log_ctas;
    return dim3(n > INT_MAX ? 0u : (unsigned)n);
}
inline int cluster_of(const RowDeal &d) { return d.joint ? 1 << d.log_ctas : 1; }

__device__ __forceinline__ RowThreads row_threads(RowShared *sh, const RowDeal &d) {
    RowThreads r;
    r.sh = sh;
    r.lane = threadIdx.x % 32;
    r.warp = threadIdx.x / 32;
    r.warps = d.rows > 1 ? 1 : d.threads / 32;
    r.ctas = d.joint ? 1u << d.log_ctas : 1u;
    r.rank = blockIdx.x & ((1u << d.log_ctas) - 1);  // in a cluster, too
    r.place = 0;
    r.t = d.rows > 1 ? (int64_t)blockIdx.x * d.rows + r.warp : blockIdx.x >> d.log_ctas;
    cluster_begin(r.ctas);
    return r;
}
// The place of a thread's first chunk among the values of its row: a warp's chunks are side by side.
template <bool kVec, int kChunks>
__device__ __forceinline__ Place<kVec> place_of(const RowThreads &r, int D) {
    const int warp = r.warps == 1 ? 0 : (int)r.rank * r.warps + r.warp;
    return Place<kVec>{warp * kChunks * kTile + r.lane * (kVec ? kWide : 1), D};
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
