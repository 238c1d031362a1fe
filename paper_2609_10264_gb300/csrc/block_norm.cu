// What lies between two blocks (pvmvmd_block_norm): norm, gate and residual, and the next
// block's norm, in one pass over a row that stays in registers.
#include "rows.cuh"

namespace pv {
namespace {

struct NormArgs {
    NormJob j;
    RowDeal d;
};

// n = norm(x) in place, for all of a thread's chunks.  Values outside the row are 0 and stay out of the
// sums.
template <bool kVec, int kChunks>
__device__ __forceinline__ void norm(RowThreads &r, const pvmvmd_norm &n, int threads, int D, float (&x)[kChunks][kWide]) {
    if (n.kind == PVMVMD_NORM_LAYER) {
        Pair s{0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int e = 0; e < kWide; ++e) add_term(s, x[c][e], 0.0f);
        const Pair m = mean_of(row_sum(r, s), (float)D);
        const float mu = __fadd_rn(m.h, m.l);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const Place<kVec> p = place_of<kVec>(r, threads, c, kChunks, D);
#pragma unroll
            for (int e = 0; e < kWide; ++e) x[c][e] = p.in(e) ? __fsub_rn(x[c][e], mu) : 0.0f;
        }
    }
    Pair s{0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int e = 0; e < kWide; ++e) add_square(s, x[c][e]);
    const float inv = inverse_root(mean_of(row_sum(r, s), (float)D), n.eps);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const Place<kVec> p = place_of<kVec>(r, threads, c, kChunks, D);
        float v[kWide];
#pragma unroll
        for (int e = 0; e < kWide; ++e) x[c][e] = __fmul_rn(x[c][e], inv);
        if (n.weight_dev) {
            unpack(load_raw<kVec>(n.weight_dev, n.type, p), n.type, v);
#pragma unroll
            for (int e = 0; e < kWide; ++e) x[c][e] = __fmul_rn(x[c][e], __fadd_rn(v[e], n.weight_add));
        } else if (n.weight_add != 0.0f) {
#pragma unroll
            for (int e = 0; e < kWide; ++e) x[c][e] = __fmul_rn(x[c][e], __fadd_rn(1.0f, n.weight_add));
        }
        if (n.bias_dev) {
            unpack(load_raw<kVec>(n.bias_dev, n.type, p), n.type, v);
#pragma unroll
            for (int e = 0; e < kWide; ++e) x[c][e] = p.in(e) ? __fadd_rn(x[c][e], v[e]) : 0.0f;
        }
    }
}

template <bool kVec, int kChunks>
__global__ void __launch_bounds__(kRowThreadsMost, kChunks == 4 ? 1 : 2)
    k_block_norm(const __grid_constant__ NormArgs a) {
    follow();
    const NormJob &j = a.j;
    __shared__ RowShared sh;
    RowThreads r = row_threads(&sh, a.d);
    cluster_begin(r.ctas);
    const int threads = a.d.threads, D = j.D;
    const int64_t t = a.d.rows > 1 ? (int64_t)blockIdx.x * a.d.rows + r.warp : blockIdx.x / r.ctas;
    if (t >= j.T) return;  // (warps of several rows have no exchanges)
    Raw y[kChunks], g[kChunks], s[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const Place<kVec> p = place_of<kVec>(r, threads, c, kChunks, D);
        if (j.has_y) y[c] = load_raw<kVec>(row_of(j.y, t), j.y.type, p);
        if (j.has_residual) s[c] = load_raw<kVec>(row_of(j.residual, t), j.residual.type, p);
        if (j.has_gate) g[c] = load_raw<kVec>(row_of(j.gate, t), j.gate.type, p);
    }
    float x[kChunks][kWide];
    if (j.has_y) {
        const float c0 = row_scale(j.y, t);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            read<kVec>(y[c], j.y, c0, place_of<kVec>(r, threads, c, kChunks, D), x[c]);
        if (j.post.kind) norm<kVec, kChunks>(r, j.post, threads, D, x);
    }
    const float gc = j.has_gate ? row_scale(j.gate, t) : 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const Place<kVec> p = place_of<kVec>(r, threads, c, kChunks, D);
        if (j.has_y) {
            if (j.has_gate) {
                float v[kWide];
                read<kVec>(g[c], j.gate, gc, p, v);
#pragma unroll
                for (int e = 0; e < kWide; ++e) x[c][e] = __fmul_rn(x[c][e], v[e]);
            }
#pragma unroll
            for (int e = 0; e < kWide; ++e) x[c][e] = __fmul_rn(x[c][e], j.branch_scale);
        }
        if (j.has_residual) {
            float v[kWide];
            unpack(s[c], j.residual.type, v);
#pragma unroll
            for (int e = 0; e < kWide; ++e) {
                const float q = __fmul_rn(v[e], j.residual_scale);
                x[c][e] = j.has_y ? __fadd_rn(q, x[c][e]) : q;
            }
        }
        if (j.residual_out.data_dev) write<kVec>(j.residual_out, t, p, x[c], 1.0f);
        // what lies outside the row is 0 from here on (a scale that is not finite made it NaN)
#pragma unroll
        for (int e = 0; e < kWide; ++e)
            if (!p.in(e)) x[c][e] = 0.0f;
    }
    if (j.out.data_dev) {
        if (j.pre.kind) norm<kVec, kChunks>(r, j.pre, threads, D, x);
        float m = j.out.scale;
        if (j.out.token_scale_dev) {
            uint32_t big = 0;
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
#pragma unroll
                for (int e = 0; e < kWide; ++e) big = max(big, __float_as_uint(x[c][e]) & 0x7fffffffu);
            float step;
            m = dynamic_scale(j.out, row_max(r, big), step);
            if (r.lane == 0 && r.rank == 0 && (r.warps == 1 || r.warp == 0)) j.out.token_scale_dev[t] = step;
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            write<kVec>(j.out, t, place_of<kVec>(r, threads, c, kChunks, D), x[c], m);
    }
    row_end(r);
}

template <bool kVec>
cudaError_t launch_vec(const NormArgs &a, cudaStream_t s) {
    const RowDeal &d = a.d;
    const dim3 grid((unsigned)(((int64_t)a.j.T + d.rows - 1) / d.rows * d.ctas));
    switch (d.chunks) {
        case 1: return launch_cluster(k_block_norm<kVec, 1>, grid, d.ctas, d.threads, 0, s, a);
        case 2: return launch_cluster(k_block_norm<kVec, 2>, grid, d.ctas, d.threads, 0, s, a);
        default: return launch_cluster(k_block_norm<kVec, 4>, grid, d.ctas, d.threads, 0, s, a);
    }
}

bool whole16(const pvmvmd_norm &n) {
    return !n.kind || (pv::whole16(n.weight_dev, 0, n.type) && pv::whole16(n.bias_dev, 0, n.type));
}

}  // namespace

cudaError_t launch_block_norm(const NormJob &j, cudaStream_t s) {
    NormArgs a{j, deal_rows(j.T, j.D)};
    const bool vec = j.D % kWide == 0 && (!j.has_y || whole16(j.y)) && (!j.has_gate || whole16(j.gate)) &&
                     (!j.has_residual || whole16(j.residual)) && whole16(j.residual_out) && whole16(j.out) &&
                     whole16(j.post) && whole16(j.pre);
    return vec ? launch_vec<true>(a, s) : launch_vec<false>(a, s);
}

}  // namespace pv
