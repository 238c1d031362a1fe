// What lies between two blocks (pvmvmd_block_norm): norm, gate and residual, and the next
// block's norm, in one pass over a row that stays in registers.
#include "rows.cuh"

namespace pv {
namespace {

struct NormArgs {
    NormJob j;
    RowDeal d;
    Pair inverse;  // 1 / D
};

// n = norm(x) in place, for all of a thread's chunks.  Values outside the row must be 0 at the call (and are
// anything after it).
template <bool kVec, int kChunks>
__device__ __forceinline__ void norm(RowThreads &r, const pvmvmd_norm &n, Pair inverse, const Place<kVec> &at,
                                     Two (&x)[kChunks][kTwos]) {
    if (n.kind == PVMVMD_NORM_LAYER) {
        Pairs s{both(0.0f), both(0.0f)};
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < kTwos; ++i) add_terms(s, x[c][i]);
        const Pair m = mean_of(row_sum(r, join(s)), inverse);
        const Two mu = both(__fadd_rn(m.h, m.l));
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[c][i] = sub2(x[c][i], mu);
            outside_zero<kVec>(at.chunk(c), x[c]);
        }
    }
    Pairs s{both(0.0f), both(0.0f)};
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < kTwos; ++i) add_squares(s, x[c][i]);
    // (the weights are on their way meanwhile)
    Raw w[kChunks];
    if (n.weight_dev)
#pragma unroll
        for (int c = 0; c < kChunks; ++c) w[c] = load_raw<kVec>(n.weight_dev, n.type, at.chunk(c));
    const Two inv = both(inverse_root(mean_of(row_sum(r, join(s)), inverse), n.eps));
    Two v[kTwos];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
#pragma unroll
        for (int i = 0; i < kTwos; ++i) x[c][i] = mul2(x[c][i], inv);
        if (n.weight_dev) {
            unpack(w[c], n.type, v);
            if (n.weight_add != 0.0f)
#pragma unroll
                for (int i = 0; i < kTwos; ++i) v[i] = add2(v[i], both(n.weight_add));
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[c][i] = mul2(x[c][i], v[i]);
        } else if (n.weight_add != 0.0f) {
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[c][i] = mul2(x[c][i], both(__fadd_rn(1.0f, n.weight_add)));
        }
        if (n.bias_dev) {
            unpack(load_raw<kVec>(n.bias_dev, n.type, at.chunk(c)), n.type, v);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[c][i] = add2(x[c][i], v[i]);
        }
    }
}

// kY, kR, kO: the kinds of y (and a gate), of the residual and its output, and of out; kGate: there may be a
// gate.
template <bool kVec, int kChunks, Kind kY, Kind kR, Kind kO, bool kGate>
__global__ void __launch_bounds__(kRowThreadsMost, kChunks == 4 ? 1 : 2)
    k_block_norm(const __grid_constant__ NormArgs a) {
    follow();
    const NormJob &j = a.j;
    __shared__ RowShared sh;
    RowThreads r = row_threads(&sh, a.d);
    const int64_t t = r.t;
    if (t >= j.T) return;  // (warps of several rows have no exchanges)
    const int yt = known<kY>(j.y.type), rt = known<kR>(j.residual.type), qt = known<kR>(j.residual_out.type),
              ot = known<kO>(j.out.type), gt = j.gate.type;
    const Place<kVec> at = place_of<kVec, kChunks>(r, j.D);
    Raw y[kChunks], g[kChunks], s[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (j.has_y) y[c] = load_raw<kVec>(row_of(j.y, yt, t), yt, at.chunk(c));
        if (j.has_residual) s[c] = load_raw<kVec>(row_of(j.residual, rt, t), rt, at.chunk(c));
        if (kGate && j.has_gate) g[c] = load_raw<kVec>(row_of(j.gate, gt, t), gt, at.chunk(c));
    }
    Two x[kChunks][kTwos];
    if (j.has_y) {
        const float c0 = row_scale(j.y, t);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) read<kVec>(y[c], j.y, yt, c0, at.chunk(c), x[c]);
        if (j.post.kind) norm<kVec, kChunks>(r, j.post, a.inverse, at, x);
    }
    const float gc = kGate && j.has_gate ? row_scale(j.gate, t) : 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        Two v[kTwos];
        if (j.has_y) {
            if (kGate && j.has_gate) {
                read<kVec>(g[c], j.gate, gt, gc, at.chunk(c), v);
#pragma unroll
                for (int i = 0; i < kTwos; ++i) x[c][i] = mul2(x[c][i], v[i]);
            }
#pragma unroll
            for (int i = 0; i < kTwos; ++i) x[c][i] = mul2(x[c][i], both(j.branch_scale));
        }
        if (j.has_residual) {
            unpack(s[c], rt, v);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) {
                v[i] = mul2(v[i], both(j.residual_scale));
                x[c][i] = j.has_y ? add2(v[i], x[c][i]) : v[i];
            }
        }
        if (j.residual_out.data_dev) write<kVec>(j.residual_out, qt, t, at.chunk(c), x[c], Step{1.0f, false});
        // what lies outside the row is 0 from here on (a bias, or a scale that is not finite, made it another value)
        outside_zero<kVec>(at.chunk(c), x[c]);
    }
    if (j.out.data_dev) {
        if (j.pre.kind) norm<kVec, kChunks>(r, j.pre, a.inverse, at, x);
        Step m{j.out.scale, false};
        if (j.out.token_scale_dev) {
            float big = 0.0f;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                outside_zero<kVec>(at.chunk(c), x[c]);
#pragma unroll
                for (int i = 0; i < kTwos; ++i) big = larger(larger(big, first(x[c][i])), second(x[c][i]));
            }
            big = row_max(r, big);
            m = step_of(j.out, big);
            if (r.lane == 0 && r.rank == 0 && (r.warps == 1 || r.warp == 0)) write_step(j.out, t, big);
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) write<kVec>(j.out, ot, t, at.chunk(c), x[c], m);
    }
    row_begun(r);
}

template <bool kVec, Kind kY, Kind kR, Kind kO, bool kGate>
cudaError_t launch_kind(const NormArgs &a, cudaStream_t s) {
    const dim3 grid = grid_of(a.d, a.j.T);
    const int ctas = 1 << a.d.log_ctas;
    switch (a.d.chunks) {
        case 1: return launch_cluster(k_block_norm<kVec, 1, kY, kR, kO, kGate>, grid, ctas, a.d.threads, 0, s, a);
        case 2: return launch_cluster(k_block_norm<kVec, 2, kY, kR, kO, kGate>, grid, ctas, a.d.threads, 0, s, a);
        default: return launch_cluster(k_block_norm<kVec, 4, kY, kR, kO, kGate>, grid, ctas, a.d.threads, 0, s, a);
    }
}
// Kernels for the kinds of a model's own types, and of the field, beside the one for any: with the kinds known, 600
// instructions a thread are left of 1170.
template <Kind kY, Kind kR, Kind kO>
cudaError_t launch_gate(const NormArgs &a, cudaStream_t s) {
    return a.j.has_gate ? launch_kind<true, kY, kR, kO, true>(a, s) : launch_kind<true, kY, kR, kO, false>(a, s);
}
template <Kind kY, Kind kR>
cudaError_t launch_out(const NormArgs &a, cudaStream_t s) {
    return kind_of(a.j.out.type) == kField ? launch_gate<kY, kR, kField>(a, s) : launch_gate<kY, kR, kHalf>(a, s);
}
template <Kind kY>
cudaError_t launch_residual(const NormArgs &a, cudaStream_t s) {
    return kind_of(a.j.residual.type) == kF32 ? launch_out<kY, kF32>(a, s) : launch_out<kY, kHalf>(a, s);
}

bool whole16(const pvmvmd_norm &n) {
    return !n.kind || (pv::whole16(n.weight_dev, 0, n.type) && pv::whole16(n.bias_dev, 0, n.type));
}

}  // namespace

cudaError_t launch_block_norm(const NormJob &j, cudaStream_t s) {
    const NormArgs a{j, deal_rows(j.T, j.D), inverse_of(j.D)};
    const bool vec = j.D % kWide == 0 && (!j.has_y || whole16(j.y)) && (!j.has_gate || whole16(j.gate)) &&
                     (!j.has_residual || whole16(j.residual)) && whole16(j.residual_out) && whole16(j.out) &&
                     whole16(j.post) && whole16(j.pre);
    if (!vec) return launch_kind<false, kAny, kAny, kAny, true>(a, s);
    if (j.has_y && j.has_residual && j.out.data_dev && kind_of(j.y.type) != kF32 && kind_of(j.out.type) != kF32 &&
        (!j.residual_out.data_dev || kind_of(j.residual_out.type) == kind_of(j.residual.type)))
        return kind_of(j.y.type) == kField ? launch_residual<kField>(a, s) : launch_residual<kHalf>(a, s);
    return launch_kind<true, kAny, kAny, kAny, true>(a, s);
}

}  // namespace pv
