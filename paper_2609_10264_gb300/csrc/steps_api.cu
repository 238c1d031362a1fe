// C ABI of the client's other steps (include/pvmvmd.h): checks of arguments and the
// launches.
#include <climits>
#include <cmath>

#include "steps.h"

namespace pv {
namespace {

#define PV_CUDA(expr)                                  \
    do {                                               \
        cudaError_t e_ = (expr);                       \
        if (e_ != cudaSuccess) {                       \
            (void)cudaGetLastError();                  \
            return e_ == cudaErrorMemoryAllocation ? PVMVMD_E_NOMEM : PVMVMD_E_CUDA; \
        }                                              \
    } while (0)

bool float_type(int t) { return t == PVMVMD_BF16 || t == PVMVMD_F16 || t == PVMVMD_F32; }
bool any_type(int t) { return float_type(t) || t == PVMVMD_FIELD; }
int size_of(int t) { return t == PVMVMD_BF16 || t == PVMVMD_F16 ? 2 : 4; }

// whether two vectors of n 32-bit values share some
bool overlap(const void *a, const void *b, int n) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && (x < y ? y - x : x - y) < (uintptr_t)n * 4;
}
bool misaligned(const void *p, int size) { return reinterpret_cast<uintptr_t>(p) % size != 0; }

// T rows of D values: addresses of whole values
int check(const pvmvmd_rows &r, bool field = true) {
    if (!r.data_dev || !(field ? any_type(r.type) : float_type(r.type))) return PVMVMD_E_ARG;
    if (misaligned(r.data_dev, size_of(r.type)) || misaligned(r.token_scale_dev, 4) || misaligned(r.channel_scale_dev, 4))
        return PVMVMD_E_ARG;
    return std::isfinite(r.scale) ? PVMVMD_OK : PVMVMD_E_PARAM;
}
// (rows closer than they are long would be written by several threads at once)
int check(const pvmvmd_rows_out &o, int T, int D, bool field = true) {
    if (!o.data_dev || !(field ? any_type(o.type) : float_type(o.type))) return PVMVMD_E_ARG;
    if (misaligned(o.data_dev, size_of(o.type)) || misaligned(o.token_scale_dev, 4)) return PVMVMD_E_ARG;
    if (T > 1 && o.token < D && o.token > -(int64_t)D) return PVMVMD_E_ARG;
    if (o.type != PVMVMD_FIELD) return o.token_scale_dev ? PVMVMD_E_ARG : PVMVMD_OK;
    if (o.limit < 1 || o.limit > kMostLimit) return PVMVMD_E_PARAM;
    return o.token_scale_dev || std::isfinite(o.scale) ? PVMVMD_OK : PVMVMD_E_PARAM;
}
int check(const pvmvmd_norm &n) {
    if (n.kind != PVMVMD_NORM_RMS && n.kind != PVMVMD_NORM_LAYER) return PVMVMD_E_ARG;
    if ((n.weight_dev || n.bias_dev) && !float_type(n.type)) return PVMVMD_E_ARG;
    if (misaligned(n.weight_dev, size_of(n.type)) || misaligned(n.bias_dev, size_of(n.type))) return PVMVMD_E_ARG;
    if (!(n.eps > 0) || !std::isfinite(n.eps) || !std::isfinite(n.weight_add)) return PVMVMD_E_PARAM;
    return PVMVMD_OK;
}
int check_size(int T, int D) { return T < 0 || D < 1 || D > PVMVMD_MAX_K ? PVMVMD_E_SHAPE : PVMVMD_OK; }

}  // namespace
}  // namespace pv

int pvmvmd_block_norm(int T, int D, const pvmvmd_rows *y, const pvmvmd_norm *post, const pvmvmd_rows *gate,
                      float branch_scale, const pvmvmd_rows *residual, float residual_scale,
                      const pvmvmd_rows_out *residual_out, const pvmvmd_norm *pre, const pvmvmd_rows_out *out,
                      void *stream) {
    using namespace pv;
    int st = check_size(T, D);
    if (st) return st;
    if ((!y && !residual) || (!residual_out && !out) || (!y && (post || gate)) || (!out && pre)) return PVMVMD_E_ARG;
    if (!std::isfinite(branch_scale) || !std::isfinite(residual_scale)) return PVMVMD_E_PARAM;
    if (post && (st = check(*post))) return st;
    if (pre && (st = check(*pre))) return st;
    if (residual && (residual->token_scale_dev || residual->channel_scale_dev || residual->scale != 1.0f)) return PVMVMD_E_ARG;
    if (T == 0) return PVMVMD_OK;
    if (y && (st = check(*y))) return st;
    if (gate && (st = check(*gate))) return st;
    if (residual && (st = check(*residual, false))) return st;
    if (residual_out && (st = check(*residual_out, T, D, false))) return st;
    if (out && (st = check(*out, T, D))) return st;
    NormJob j{};
    j.T = T;
    j.D = D;
    j.residual_scale = residual_scale;
    j.branch_scale = branch_scale;
    if ((j.has_y = y)) j.y = *y;
    if ((j.has_gate = gate)) j.gate = *gate;
    if ((j.has_residual = residual)) j.residual = *residual;
    if (residual_out) j.residual_out = *residual_out;
    if (out) j.out = *out;
    if (post) j.post = *post;
    if (pre) j.pre = *pre;
    PV_CUDA(launch_block_norm(j, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}

int pvmvmd_glu(int T, int D, const pvmvmd_rows *gate, int act, const pvmvmd_rows *up, const pvmvmd_rows_out *out,
               void *stream) {
    using namespace pv;
    int st = check_size(T, D);
    if (st) return st;
    if (!gate || !out || act < PVMVMD_ACT_NONE || act > PVMVMD_ACT_GELU) return PVMVMD_E_ARG;
    if (T == 0) return PVMVMD_OK;
    if ((st = check(*gate)) || (up && (st = check(*up))) || (st = check(*out, T, D))) return st;
    GluJob j{};
    j.T = T;
    j.D = D;
    j.act = act;
    j.gate = *gate;
    if ((j.has_up = up)) j.up = *up;
    j.out = *out;
    PV_CUDA(launch_glu(j, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}

int pvmvmd_sample(int T, int V, const pvmvmd_rows *logits, const pvmvmd_sampling *sampling, const uint32_t *allowed_dev,
                  int64_t allowed_row, const uint32_t *random_dev, int32_t *token_dev, float *logprob_dev, void *stream) {
    using namespace pv;
    if (T < 0 || V < 1 || V > PVMVMD_MAX_V) return PVMVMD_E_SHAPE;
    if (!logits || !sampling) return PVMVMD_E_ARG;
    if (T == 0) return PVMVMD_OK;
    const int st = check(*logits);
    if (st) return st;
    if (!random_dev || !token_dev) return PVMVMD_E_ARG;
    for (const void *p : {static_cast<const void *>(random_dev), static_cast<const void *>(token_dev),
                          static_cast<const void *>(logprob_dev), static_cast<const void *>(allowed_dev),
                          static_cast<const void *>(sampling->temperature_dev), static_cast<const void *>(sampling->top_k_dev),
                          static_cast<const void *>(sampling->top_p_dev), static_cast<const void *>(sampling->min_p_dev)})
        if (misaligned(p, 4)) return PVMVMD_E_ARG;
    // (a row's CTAs read its word one after the other, some when its token is written)
    if (overlap(random_dev, token_dev, T) || overlap(random_dev, logprob_dev, T)) return PVMVMD_E_ARG;
    SampleJob j{};
    j.T = T;
    j.V = V;
    j.logits = *logits;
    j.how = *sampling;
    j.allowed = allowed_dev;
    j.allowed_row = allowed_row;
    j.random = random_dev;
    j.token = token_dev;
    j.logprob = logprob_dev;
    PV_CUDA(launch_sample(j, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}
