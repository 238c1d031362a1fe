// The gated activation of a feed-forward block (pvmvmd_glu).
//
// fp32 is bound by memory: 4096 rows of 28672 198 us (7.1 TB/s, without channel scales).  Of field elements and 16-bit types
// a value takes 50 and 29 instructions with its scales, power and quotient; they fill half of an SM's issue slots, and in the
// others all warps wait, for their loads above all: bf16 141 us (5.0 TB/s), field elements with channel scales to
// integers by a scale known ahead 239 (5.9 TB/s).  With a step a row 296: nothing is under way from a row's last load to the
// next row's first, while its maximum is taken and it is written.  One row of 14336 3.3 us.
#include "rows.cuh"

namespace pv {
namespace {

struct GluArgs {
    GluJob j;
    RowDeal d;
};

// 2 sqrt(2 / pi) log2 e, and 0.044715 of it
constexpr double kC = 1.5957691216057308 * 1.4426950408889634;
constexpr float kGelu1 = (float)kC, kGelu3 = (float)(0.044715 * kC);

__device__ __forceinline__ float near_inverse(float b) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(b));
    return y;
}
// x / (1 + power), rounded as the quotient of two numbers is (Markstein, IBM J. Res. Dev. 34, 1990): y the
// inverse to half a step, q the quotient to a step, and its rest r, exact, over b.  That can fail where b's
// bits are all ones and x is a power of two, which no x has here; where b's inverse is below 2^-126; and for
// infinities.  So it serves what |x| is not above `most` of, for which tests compare every one of the
// numbers of 32 bits.  (A third of the instructions of the division for any numbers, which
// were 14 of 65 a value.)
__device__ __forceinline__ Two over_one_plus(Two x, Two power) {
    const Two b = add2(both(1.0f), power), minus_b = sub2(both(-1.0f), power);
    Two y = two(near_inverse(first(b)), near_inverse(second(b)));
    y = fma2(y, fma2(minus_b, y, both(1.0f)), y);
    const Two q = mul2(x, y);
    return fma2(fma2(minus_b, q, x), y, q);
}
__device__ __forceinline__ Two over_one_plus_any(Two x, Two power) {
    const Two b = add2(both(1.0f), power);
    return two(__fdiv_rn(first(x), first(b)), __fdiv_rn(second(x), second(b)));
}
template <int kAct>
__device__ __forceinline__ Two distance(Two v) {
    return kAct == PVMVMD_ACT_GELU ? mul2(add2(mul2(mul2(v, v), both(kGelu3)), both(kGelu1)), v) : mul2(v, both(kLog2e));
}
template <int kAct>
__device__ __noinline__ unsigned long long activate_any(unsigned long long x) {
    return over_one_plus_any(Two{x}, power(distance<kAct>(Two{x}))).v;
}
// (Where a thread has a larger value, its eight go through the divisions one after the other: 4096 rows of 14336 bf16 values
// take 67 us with GELU, 83 where one value in a thousand is above 10 and 118 where one in a hundred is; with SiLU and 80 63, 78
// and 110; sigmoid, which always does, 76.)
template <int kAct>
__device__ __forceinline__ void over_one_plus_all(Two (&x)[kTwos], float most) {
    float big = 0.0f;
#pragma unroll
    for (int i = 0; i < kTwos; ++i) big = larger(larger(big, first(x[i])), second(x[i]));
    if (big <= most) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = over_one_plus(x[i], power_near(distance<kAct>(x[i])));  // (at 126 or 125, 1 + 2^-d is 1)
    } else {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i].v = activate_any<kAct>(x[i].v);
    }
}

__device__ __forceinline__ void activate(Two (&x)[kTwos], int act) {
    if (act == PVMVMD_ACT_SILU) {
        over_one_plus_all<PVMVMD_ACT_SILU>(x, 80.0f);
    } else if (act == PVMVMD_ACT_GELU) {
        over_one_plus_all<PVMVMD_ACT_GELU>(x, 10.0f);
    } else if (act == PVMVMD_ACT_SIGMOID) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) {
            const Two v = over_one_plus_any(both(1.0f), power(mul2(x[i], both(kLog2e))));
            x[i] = two(first(x[i]) == first(x[i]) ? first(v) : first(x[i]), second(x[i]) == second(x[i]) ? second(v) : second(x[i]));
        }
    } else if (act == PVMVMD_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i)
            x[i] = two(first(x[i]) < 0.0f ? 0.0f : first(x[i]), second(x[i]) < 0.0f ? 0.0f : second(x[i]));
    }
}

// A thread's chunks of a row; the row's largest value only where integers have a step of their own.
// kX: the type of gate and up; kO: of out.
template <bool kVec, int kChunks, int kX, int kO>
__global__ void __launch_bounds__(kRowThreadsMost, kChunks == 4 ? 1 : 2) k_glu(const __grid_constant__ GluArgs a) {
    follow();
    const GluJob &j = a.j;
    __shared__ RowShared sh;
    RowThreads r = row_threads(&sh, a.d);
    const int64_t t = r.t;
    if (t >= j.T) return;  // (warps of several rows have no exchanges)
    const int gt = known<kX>(j.gate.type), ut = known<kX>(j.up.type), ot = known<kO>(j.out.type);
    const Place<kVec> at = place_of<kVec, kChunks>(r, j.D);
    Raw g[kChunks], u[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        g[c] = load_raw<kVec>(row_of(j.gate, gt, t), gt, at.chunk(c));
        if (j.has_up) u[c] = load_raw<kVec>(row_of(j.up, ut, t), ut, at.chunk(c));
    }
    const float gc = row_scale(j.gate, t), uc = j.has_up ? row_scale(j.up, t) : 0.0f;
    Two x[kChunks][kTwos];
    float big = 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        read<kVec>(g[c], j.gate, gt, gc, at.chunk(c), x[c]);
        activate(x[c], j.act);
        if (j.has_up) {
            Two v[kTwos];
            read<kVec>(u[c], j.up, ut, uc, at.chunk(c), v);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[c][i] = mul2(x[c][i], v[i]);
        }
        if (j.out.token_scale_dev) {
            outside_zero<kVec>(at.chunk(c), x[c]);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) big = larger(larger(big, first(x[c][i])), second(x[c][i]));
        }
    }
    Step m{j.out.scale, false};
    if (j.out.token_scale_dev) {
        big = row_max(r, big);
        m = step_of(j.out, big);
        if (r.lane == 0 && r.rank == 0 && (r.warps == 1 || r.warp == 0)) write_step(j.out, t, big);
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) write<kVec>(j.out, ot, t, at.chunk(c), x[c], m);
    row_begun(r);
}

// One CTA a row, for rows that are too long for the registers of one: the values wait in shared memory
// for the largest of them.  (4096 x 28672 field elements to integers 296 us, 343 with the row in the
// registers of a cluster of 8; 14336 values a row 144 and 171.)  Raw values of 32 bits take so many registers
// that 512 threads, of 64 each, spill: 308 us and 157.  Those of 16 bits do not: 241 us with 512 threads, 265 with 448.
constexpr int kLongMost = 57344;
template <int kX>
constexpr int kLongThreads = kX == kField ? 448 : 512;
template <int kX>
__global__ void __launch_bounds__(kLongThreads<kX>, 2) k_glu_long(const __grid_constant__ GluArgs a) {
    follow();
    const GluJob &j = a.j;
    extern __shared__ __align__(16) float4 s_z[];  // of chunk c and half h at (2 c + h) kThreads + thread
    __shared__ RowShared sh;
    RowThreads r = row_threads(&sh, a.d);
    const int64_t t = r.t;
    const int gt = known<kX>(j.gate.type), ut = known<kX>(j.up.type);
    const void *g_row = row_of(j.gate, gt, t), *u_row = row_of(j.up, ut, t);
    const float gc = row_scale(j.gate, t), uc = j.has_up ? row_scale(j.up, t) : 0.0f;
    constexpr int kThreads = kLongThreads<kX>, kStride = kThreads * kWide;
    Place<true> p{(int)threadIdx.x * kWide, j.D};
    Raw g = load_raw<true>(g_row, gt, p), u = g;
    if (j.has_up) u = load_raw<true>(u_row, ut, p);
    float big = 0.0f;
    float4 *z = s_z + threadIdx.x;
    for (; p.any(); p.at += kStride, z += 2 * kThreads) {
        const Raw g0 = g, u0 = u;
        const Place<true> next{p.at + kStride, p.D};
        g = load_raw<true>(g_row, gt, next);
        if (j.has_up) u = load_raw<true>(u_row, ut, next);
        Two x[kTwos];
        read<true>(g0, j.gate, gt, gc, p, x);
        activate(x, j.act);
        if (j.has_up) {
            Two v[kTwos];
            read<true>(u0, j.up, ut, uc, p, v);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[i] = mul2(x[i], v[i]);
        }
#pragma unroll
        for (int i = 0; i < kTwos; ++i) big = larger(larger(big, first(x[i])), second(x[i]));
        z[0] = make_float4(first(x[0]), second(x[0]), first(x[1]), second(x[1]));
        z[kThreads] = make_float4(first(x[2]), second(x[2]), first(x[3]), second(x[3]));
    }
    big = row_max(r, big);
    const Step m = step_of(j.out, big);
    if (threadIdx.x == 0) write_step(j.out, t, big);
    z = s_z + threadIdx.x;
    for (p.at = (int)threadIdx.x * kWide; p.any(); p.at += kStride, z += 2 * kThreads) {
        const float4 lo = z[0], hi = z[kThreads];
        const Two x[kTwos] = {two(lo.x, lo.y), two(lo.z, lo.w), two(hi.x, hi.y), two(hi.z, hi.w)};
        write<true>(j.out, PVMVMD_FIELD, t, p, x, m);
    }
}
template <int kX>
cudaError_t launch_long(GluArgs a, cudaStream_t s) {
    constexpr int kStride = kLongThreads<kX> * kWide;
    a.d = RowDeal{kLongThreads<kX>, 1, 0, 1, true};
    const size_t smem = (size_t)((a.j.D + kStride - 1) / kStride) * kStride * sizeof(float);
    const cudaError_t e = func_attr(reinterpret_cast<const void *>(k_glu_long<kX>), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    kLongMost * (int)sizeof(float));
    if (e != cudaSuccess) return e;
    return launch_dependent(k_glu_long<kX>, grid_of(a.d, a.j.T), kLongThreads<kX>, smem, s, a);
}

template <bool kVec, int kX, int kO>
cudaError_t launch_types(const GluArgs &a, cudaStream_t s) {
    const dim3 grid = grid_of(a.d, a.j.T);
    const int ctas = cluster_of(a.d);
    switch (a.d.chunks) {
        case 1: return launch_cluster(k_glu<kVec, 1, kX, kO>, grid, ctas, a.d.threads, 0, s, a);
        case 2: return launch_cluster(k_glu<kVec, 2, kX, kO>, grid, ctas, a.d.threads, 0, s, a);
        default: return launch_cluster(k_glu<kVec, 4, kAny, kAny>, grid, ctas, a.d.threads, 0, s, a);
    }
}
// Kernels for the types that a model has together (a field element or one type of 16 bits in, and out), beside the one
// for any.
template <int kX>
cudaError_t launch_out(const GluArgs &a, cudaStream_t s) {
    switch (a.j.out.type) {
        case kField: return launch_types<true, kX, kField>(a, s);
        case kBf16: return launch_types<true, kX, kX == kField ? kBf16 : kX == kBf16 ? kBf16 : kAny>(a, s);
        case kF16: return launch_types<true, kX, kX == kField ? kF16 : kX == kF16 ? kF16 : kAny>(a, s);
        default: return launch_types<true, kAny, kAny>(a, s);
    }
}

}  // namespace

cudaError_t launch_glu(const GluJob &j, cudaStream_t s) {
    const GluArgs a{j, deal_rows(j.T, j.D, j.out.token_scale_dev != nullptr)};
    const bool vec = j.D % kWide == 0 && whole16(j.gate) && (!j.has_up || whole16(j.up)) && whole16(j.out);
    if (!vec) return launch_types<false, kAny, kAny>(a, s);
    if (j.has_up && j.up.type != j.gate.type) return launch_types<true, kAny, kAny>(a, s);
    const bool is_long = j.T >= kSms && j.D > 8192 && j.D <= kLongMost && j.out.token_scale_dev;
    switch (j.gate.type) {
        case kField: return is_long ? launch_long<kField>(a, s) : launch_out<kField>(a, s);
        case kBf16: return is_long ? launch_long<kBf16>(a, s) : launch_out<kBf16>(a, s);
        case kF16: return is_long ? launch_long<kF16>(a, s) : launch_out<kF16>(a, s);
        default: return launch_types<true, kAny, kAny>(a, s);
    }
}

}  // namespace pv
