// The gated activation of a feed-forward block (pvmvmd_glu).
#include "rows.cuh"

namespace pv {
namespace {

struct GluArgs {
    GluJob j;
    RowDeal d;
};

__device__ __forceinline__ void activate(Two (&x)[kTwos], int act) {
    constexpr float kLog2e = 1.442695041f;
    // 2 sqrt(2 / pi) log2 e, and 0.044715 of it
    constexpr double kC = 1.5957691216057308 * 1.4426950408889634;
    if (act == PVMVMD_ACT_NONE) return;
    if (act == PVMVMD_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[i] = two(first(x[i]) < 0.0f ? 0.0f : first(x[i]), second(x[i]) < 0.0f ? 0.0f : second(x[i]));
        return;
    }
#pragma unroll
    for (int i = 0; i < kTwos; ++i) {
        Two d;
        if (act == PVMVMD_ACT_GELU)
            d = mul2(add2(mul2(mul2(x[i], x[i]), both((float)(0.044715 * kC))), both((float)kC)), x[i]);
        else
            d = mul2(x[i], both(kLog2e));
        d = one_plus_exp(d);
        if (act == PVMVMD_ACT_SIGMOID)
            x[i] = two(first(x[i]) == first(x[i]) ? __fdiv_rn(1.0f, first(d)) : first(x[i]),
                       second(x[i]) == second(x[i]) ? __fdiv_rn(1.0f, second(d)) : second(x[i]));
        else
            x[i] = two(__fdiv_rn(first(x[i]), first(d)), __fdiv_rn(second(x[i]), second(d)));
    }
}

// A thread's chunks of a row; the row's largest value only where integers have a step of their own.
// kX: the kind of gate and up; kO: of out.
template <bool kVec, int kChunks, Kind kX, Kind kO>
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

template <bool kVec, Kind kX, Kind kO>
cudaError_t launch_kind(const GluArgs &a, cudaStream_t s) {
    const dim3 grid = grid_of(a.d, a.j.T);
    const int ctas = 1 << a.d.log_ctas;
    switch (a.d.chunks) {
        case 1: return launch_cluster(k_glu<kVec, 1, kX, kO>, grid, ctas, a.d.threads, 0, s, a);
        case 2: return launch_cluster(k_glu<kVec, 2, kX, kO>, grid, ctas, a.d.threads, 0, s, a);
        default: return launch_cluster(k_glu<kVec, 4, kX, kO>, grid, ctas, a.d.threads, 0, s, a);
    }
}
template <Kind kX>
cudaError_t launch_out(const GluArgs &a, cudaStream_t s) {
    return kind_of(a.j.out.type) == kField ? launch_kind<true, kX, kField>(a, s) : launch_kind<true, kX, kHalf>(a, s);
}

}  // namespace

cudaError_t launch_glu(const GluJob &j, cudaStream_t s) {
    const GluArgs a{j, deal_rows(j.T, j.D)};
    const bool vec = j.D % kWide == 0 && whole16(j.gate) && (!j.has_up || whole16(j.up)) && whole16(j.out);
    if (!vec) return launch_kind<false, kAny, kAny>(a, s);
    const Kind x = kind_of(j.gate.type);
    if (x != kF32 && kind_of(j.out.type) != kF32 && (!j.has_up || kind_of(j.up.type) == x))
        return x == kField ? launch_out<kField>(a, s) : launch_out<kHalf>(a, s);
    return launch_kind<true, kAny, kAny>(a, s);
}

}  // namespace pv
