// What lies between two blocks (pvmvmd_block_norm): norm, gate and residual, and the next
// block's norm, in one pass over a row that stays in registers.
//
// Bound by memory where rows are many (8192 rows of 8192 field elements, bf16 residual, to integers with a step a row
// 154 us, 5.2 TB/s; of 4096, 71 us, 5.7 TB/s) and by the latency of a load, two exchanges and a store where they
// are few (one row of 4096 3.6 us).  8192 rows of 8192 in fp32 179 us (6.0 TB/s), in bf16 99 (5.4 TB/s).
// A call with a row, scale or weight off the 16-byte boundaries goes value by value, by the kernel for any types: 67
// instructions a value in half of the issue slots, and loads of 4 bytes that are waited for in the others (333 rows of 5001
// in fp32 15 us, 1.8 TB/s).
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
        const Two mu = both(rounded_mean(row_sum(r, join(s)), (float)at.D, inverse.h));
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

// kY, kR, kO, kG: the types of y, of the residual and its output, of out, and of the gate (kNone: there is
// none).  kMost: threads at most.  With a gate 64 registers a thread, which let two CTAs of 512 run, spill a few; CTAs of up to
// 224 have 72 (4096 gated rows of 8192 94 us with 64 and 116 with 72, where one CTA runs; of 2560 31.4 and 28.9).
constexpr int kNone = -1, kFewThreads = 224;
template <bool kVec, int kChunks, int kY, int kR, int kO, int kG, int kMost = kRowThreadsMost>
__global__ void __launch_bounds__(kMost, kMost == kFewThreads ? 4 : kChunks == 4 ? 1 : 2)
    k_block_norm(const __grid_constant__ NormArgs a) {
    follow();
    const NormJob &j = a.j;
    __shared__ RowShared sh;
    RowThreads r = row_threads(&sh, a.d);
    const int64_t t = r.t;
    if (t >= j.T) return;  // (warps of several rows have no exchanges)
    const int yt = known<kY>(j.y.type), rt = known<kR>(j.residual.type), qt = known<kR>(j.residual_out.type),
              ot = known<kO>(j.out.type), gt = known<kG>(j.gate.type);
    const Place<kVec> at = place_of<kVec, kChunks>(r, j.D);
    Raw y[kChunks], g[kChunks], s[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (j.has_y) y[c] = load_raw<kVec>(row_of(j.y, yt, t), yt, at.chunk(c));
        if (j.has_residual) s[c] = load_raw<kVec>(row_of(j.residual, rt, t), rt, at.chunk(c));
        if (kG != kNone && j.has_gate) g[c] = load_raw<kVec>(row_of(j.gate, gt, t), gt, at.chunk(c));
    }
    Two x[kChunks][kTwos];
    if (j.has_y) {
        const float c0 = row_scale(j.y, t);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) read<kVec>(y[c], j.y, yt, c0, at.chunk(c), x[c]);
        if (j.post.kind) norm<kVec, kChunks>(r, j.post, a.inverse, at, x);
    }
    const float gc = kG != kNone && j.has_gate ? row_scale(j.gate, t) : 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        Two v[kTwos];
        if (j.has_y) {
            if (kG != kNone && j.has_gate) {
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

template <bool kVec, int kY, int kR, int kO, int kG>
cudaError_t launch_types(const NormArgs &a, cudaStream_t s) {
    const dim3 grid = grid_of(a.d, a.j.T);
    const int ctas = cluster_of(a.d);
    switch (a.d.chunks) {
        case 1: return launch_cluster(k_block_norm<kVec, 1, kY, kR, kO, kG>, grid, ctas, a.d.threads, 0, s, a);
        case 2:
            if constexpr (kG > kAny)
                if (a.d.threads <= kFewThreads)
                    return launch_cluster(k_block_norm<kVec, 2, kY, kR, kO, kG, kFewThreads>, grid, ctas, a.d.threads, 0, s, a);
            return launch_cluster(k_block_norm<kVec, 2, kY, kR, kO, kG>, grid, ctas, a.d.threads, 0, s, a);
        default: return launch_cluster(k_block_norm<kVec, 4, kAny, kAny, kAny, kAny>, grid, ctas, a.d.threads, 0, s, a);
    }
}
// Kernels for the types that a model has together, beside the one for any: with the types known, 800
// instructions a thread are left of 1170 (8192 x 8192 201 us without, 155 with).  kH: the model's own, of 16 bits; y may be a field element, the residual of
// 32 bits, and out a field element.
template <int kH, int kY, int kR>
cudaError_t launch_out(const NormArgs &a, cudaStream_t s) {
    if (a.j.out.type == kField)
        return a.j.has_gate ? launch_types<true, kY, kR, kField, kH>(a, s) : launch_types<true, kY, kR, kField, kNone>(a, s);
    return a.j.has_gate ? launch_types<true, kY, kR, kH, kH>(a, s) : launch_types<true, kY, kR, kH, kNone>(a, s);
}
template <int kH>
cudaError_t launch_model(const NormArgs &a, cudaStream_t s) {
    if (a.j.y.type == kField)
        return a.j.residual.type == kF32 ? launch_out<kH, kField, kF32>(a, s) : launch_out<kH, kField, kH>(a, s);
    return a.j.residual.type == kF32 ? launch_out<kH, kH, kF32>(a, s) : launch_out<kH, kH, kH>(a, s);
}
// Whether a call's types are those of a model of type h.
bool of_model(const NormJob &j, int h) {
    return j.has_y && j.has_residual && j.out.data_dev && (j.y.type == h || j.y.type == kField) &&
           (j.residual.type == h || j.residual.type == kF32) && (j.out.type == h || j.out.type == kField) && (!j.has_gate || j.gate.type == h) &&
           (!j.residual_out.data_dev || j.residual_out.type == j.residual.type);
}

bool whole16(const pvmvmd_norm &n) {
    return !n.kind || (pv::whole16(n.weight_dev, 0, n.type) && pv::whole16(n.bias_dev, 0, n.type));
}

}  // namespace

cudaError_t launch_block_norm(const NormJob &j, cudaStream_t s) {
    const NormArgs a{j, deal_rows(j.T, j.D, true), inverse_of(j.D)};
    const bool vec = j.D % kWide == 0 && (!j.has_y || whole16(j.y)) && (!j.has_gate || whole16(j.gate)) &&
                     (!j.has_residual || whole16(j.residual)) && whole16(j.residual_out) && whole16(j.out) &&
                     whole16(j.post) && whole16(j.pre);
    if (vec && of_model(j, kBf16)) return launch_model<kBf16>(a, s);
    if (vec && of_model(j, kF16)) return launch_model<kF16>(a, s);
    return vec ? launch_types<true, kAny, kAny, kAny, kAny>(a, s) : launch_types<false, kAny, kAny, kAny, kAny>(a, s);
}

}  // namespace pv
