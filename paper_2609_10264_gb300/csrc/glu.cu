// The gated activation of a feed-forward block (pvmvmd_glu).
#include "rows.cuh"

namespace pv {
namespace {

struct GluArgs {
    GluJob j;
    RowDeal d;
};

__device__ __forceinline__ float activate(float x, int act) {
    constexpr float kLog2e = 1.442695041f;
    // 2 sqrt(2 / pi) log2 e, and 0.044715 of it
    constexpr double kC = 1.5957691216057308 * 1.4426950408889634;
    switch (act) {
        case PVMVMD_ACT_RELU: return x < 0.0f ? 0.0f : x;
        case PVMVMD_ACT_SIGMOID: return x == x ? __fdiv_rn(1.0f, one_plus_exp(__fmul_rn(x, kLog2e))) : x;
        case PVMVMD_ACT_SILU: return __fdiv_rn(x, one_plus_exp(__fmul_rn(x, kLog2e)));
        case PVMVMD_ACT_GELU: {
            const float u = __fadd_rn(__fmul_rn(__fmul_rn(x, x), (float)(0.044715 * kC)), (float)kC);
            return __fdiv_rn(x, one_plus_exp(__fmul_rn(u, x)));
        }
        default: return x;
    }
}

// A thread's chunks of a row; the row's largest value only where integers have a step of their own.
template <bool kVec, int kChunks>
__global__ void __launch_bounds__(kRowThreadsMost, kChunks == 4 ? 1 : 2) k_glu(const __grid_constant__ GluArgs a) {
    follow();
    const GluJob &j = a.j;
    __shared__ RowShared sh;
    RowThreads r = row_threads(&sh, a.d);
    cluster_begin(r.ctas);
    const int threads = a.d.threads, D = j.D;
    const int64_t t = a.d.rows > 1 ? (int64_t)blockIdx.x * a.d.rows + r.warp : blockIdx.x / r.ctas;
    if (t >= j.T) return;  // (warps of several rows have no exchanges)
    Raw g[kChunks], u[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const Place<kVec> p = place_of<kVec>(r, threads, c, kChunks, D);
        g[c] = load_raw<kVec>(row_of(j.gate, t), j.gate.type, p);
        if (j.has_up) u[c] = load_raw<kVec>(row_of(j.up, t), j.up.type, p);
    }
    const float gc = row_scale(j.gate, t), uc = j.has_up ? row_scale(j.up, t) : 0.0f;
    float x[kChunks][kWide];
    uint32_t big = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const Place<kVec> p = place_of<kVec>(r, threads, c, kChunks, D);
        read<kVec>(g[c], j.gate, gc, p, x[c]);
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[c][e] = activate(x[c][e], j.act);
        if (j.has_up) {
            float v[kWide];
            read<kVec>(u[c], j.up, uc, p, v);
#pragma unroll
            for (int e = 0; e < kWide; ++e) x[c][e] = __fmul_rn(x[c][e], v[e]);
        }
#pragma unroll
        for (int e = 0; e < kWide; ++e)
            if (p.in(e)) big = max(big, __float_as_uint(x[c][e]) & 0x7fffffffu);
    }
    float m = j.out.scale;
    if (j.out.token_scale_dev) {
        float step;
        m = dynamic_scale(j.out, row_max(r, big), step);
        if (r.lane == 0 && r.rank == 0 && (r.warps == 1 || r.warp == 0)) j.out.token_scale_dev[t] = step;
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) write<kVec>(j.out, t, place_of<kVec>(r, threads, c, kChunks, D), x[c], m);
    row_end(r);
}

template <bool kVec>
cudaError_t launch_vec(const GluArgs &a, cudaStream_t s) {
    const RowDeal &d = a.d;
    const dim3 grid((unsigned)(((int64_t)a.j.T + d.rows - 1) / d.rows * d.ctas));
    switch (d.chunks) {
        case 1: return launch_cluster(k_glu<kVec, 1>, grid, d.ctas, d.threads, 0, s, a);
        case 2: return launch_cluster(k_glu<kVec, 2>, grid, d.ctas, d.threads, 0, s, a);
        default: return launch_cluster(k_glu<kVec, 4>, grid, d.ctas, d.threads, 0, s, a);
    }
}

}  // namespace

cudaError_t launch_glu(const GluJob &j, cudaStream_t s) {
    const GluArgs a{j, deal_rows(j.T, j.D)};
    const bool vec = j.D % kWide == 0 && whole16(j.gate) && (!j.has_up || whole16(j.up)) && whole16(j.out);
    return vec ? launch_vec<true>(a, s) : launch_vec<false>(a, s);
}

}  // namespace pv
