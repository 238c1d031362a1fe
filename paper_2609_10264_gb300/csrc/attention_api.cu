// C ABI of the client's attention (include/pvmvmd.h): checks of arguments and the
// launches.
#include <algorithm>
#include <climits>
#include <cmath>

#include "attention.h"
#include "kv.cuh"

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
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// strides of rows that are read 16 bytes at a time, 16-bit elements
bool rows16(int64_t a, int64_t b) { return a % 8 == 0 && b % 8 == 0; }

int check_rope(const pvmvmd_rope_view *r, int D) {
    if (!r->turns_dev) return PVMVMD_E_ARG;
    return r->rot < 2 || r->rot % 2 || r->rot > D ? PVMVMD_E_SHAPE : PVMVMD_OK;
}

int view(const pvmvmd_kv_pool *p, const pvmvmd_kv_batch *b, KvView &v) {
    if (!p || !b || !p->K_dev || !p->V_dev || !b->table_dev || !b->lens_dev) return PVMVMD_E_ARG;
    if (p->type != PVMVMD_BF16 && p->type != PVMVMD_F16) return PVMVMD_E_ARG;
    if (!aligned16(p->K_dev) || !aligned16(p->V_dev) || !rows16(p->k_page, p->k_slot) || !rows16(p->v_page, p->v_slot) ||
        !rows16(p->k_head, p->v_head))
        return PVMVMD_E_ARG;
    if (p->pages < 1 || p->page_size < 1 || p->heads < 1 || p->dim < 8 || p->dim > PVMVMD_MAX_HEAD || p->dim % 8)
        return PVMVMD_E_SHAPE;
    if (b->B < 1 || b->B > 65535 || p->heads > 65535 || b->T < 0 || b->max_pages < 1 || b->max_new < 0) return PVMVMD_E_SHAPE;
    if ((int64_t)b->max_pages * p->page_size > 1 << 30) return PVMVMD_E_SHAPE;  // cache indexes are ints
    v.K = static_cast<char *>(p->K_dev);
    v.V = static_cast<char *>(p->V_dev);
    v.mass = p->mass_dev;
    v.k_page = 2 * p->k_page;
    v.k_slot = 2 * p->k_slot;
    v.k_head = 2 * p->k_head;
    v.v_page = 2 * p->v_page;
    v.v_slot = 2 * p->v_slot;
    v.v_head = 2 * p->v_head;
    v.pages = p->pages;
    v.heads = p->heads;
    v.dim = p->dim;
    v.ps = FastDiv((uint32_t)p->page_size);
    v.table = b->table_dev;
    v.lens = b->lens_dev;
    v.cu = b->cu_dev;
    v.table_stride = b->table_stride;
    v.B = b->B;
    v.T = b->T;
    v.max_pages = b->max_pages;
    v.max_new = !b->cu_dev ? 1 : b->max_new ? std::min(b->max_new, b->T) : b->T;
    return PVMVMD_OK;
}
// the batch of a call that has new tokens
int check_new(const pvmvmd_kv_batch *b) { return !b->cu_dev && b->T != b->B ? PVMVMD_E_SHAPE : PVMVMD_OK; }

}  // namespace
}  // namespace pv

int pvmvmd_rope_turns(const pvmvmd_rope_params *p, uint64_t *turns) {
    if (!p || !turns) return PVMVMD_E_ARG;
    if (p->rot < 2 || p->rot % 2 || !(p->base > 0) || !std::isfinite(p->base)) return PVMVMD_E_PARAM;
    double base = p->base;
    const double s = p->factor, two_pi = 6.283185307179586476925;
    if (p->scaling != PVMVMD_ROPE_PLAIN && (!(s >= 1) || !std::isfinite(s))) return PVMVMD_E_PARAM;
    switch (p->scaling) {
        case PVMVMD_ROPE_PLAIN:
        case PVMVMD_ROPE_LINEAR: break;
        case PVMVMD_ROPE_BASE:
            if (p->rot == 2) return PVMVMD_E_PARAM;
            base *= std::pow(s, (double)p->rot / (p->rot - 2));
            break;
        case PVMVMD_ROPE_RAMP:
            if (!(p->original > 0) || !(p->fast > p->slow) || !std::isfinite(p->original) || !std::isfinite(p->fast) ||
                !std::isfinite(p->slow))
                return PVMVMD_E_PARAM;
            break;
        default: return PVMVMD_E_PARAM;
    }
    for (int i = 0; i < p->rot / 2; ++i) {
        double th = std::pow(base, -2.0 * i / p->rot);
        if (p->scaling == PVMVMD_ROPE_LINEAR) th /= s;
        if (p->scaling == PVMVMD_ROPE_RAMP) {
            double g = (p->original * th / two_pi - p->slow) / (p->fast - p->slow);
            g = g < 0 ? 0 : g > 1 ? 1 : g;
            th *= g + (1 - g) / s;
        }
        double turn = th / two_pi;
        if (!std::isfinite(turn)) return PVMVMD_E_PARAM;  // bases next to 0
        turn -= std::floor(turn);  // exact; bases below 1 turn more than once a position
        turn *= 18446744073709551616.0;
        turns[i] = turn >= 18446744073709551615.0 ? 0 : (uint64_t)turn;
    }
    return PVMVMD_OK;
}

int pvmvmd_rope(const pvmvmd_rope_view *rope, const int32_t *pos_dev, int T, int H, int D, const void *x_dev,
                int x_type, int64_t x_token, int64_t x_head, float scale, void *out_dev, int out_type,
                int64_t out_token, int64_t out_head, void *stream) {
    using namespace pv;
    if (!rope || !any_type(x_type) || !float_type(out_type)) return PVMVMD_E_ARG;
    if (T < 0 || H < 1 || D < 1) return PVMVMD_E_SHAPE;
    const int st = check_rope(rope, D);
    if (st) return st;
    if (T == 0) return PVMVMD_OK;
    if (!pos_dev || !x_dev || !out_dev) return PVMVMD_E_ARG;
    RopeJob j{};
    j.turns = rope->turns_dev;
    j.pos = pos_dev;
    j.part[0] = RopePart{x_dev, out_dev, x_token, x_head, out_token, out_head, H};
    j.T = T;
    j.dim = D;
    j.rot = rope->rot;
    j.interleaved = rope->interleaved != 0;
    j.in_type = x_type;
    j.out_type = out_type;
    j.magnitude = rope->magnitude;
    j.scale = scale;
    PV_CUDA(launch_rope(j, nullptr, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}

int pvmvmd_kv_append(const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch, const pvmvmd_rope_view *rope,
                     const int32_t *pos_dev, int in_type, float scale, const void *k_dev, int64_t k_token,
                     int64_t k_head, const void *v_dev, int64_t v_token, int64_t v_head, int Hq, const void *q_dev,
                     int64_t q_token, int64_t q_head, void *q_out_dev, int64_t q_out_token, int64_t q_out_head,
                     void *stream) {
    using namespace pv;
    KvView kv;
    int st = view(pool, batch, kv);
    if (!st) st = check_new(batch);
    if (!st && rope) st = check_rope(rope, kv.dim);
    if (st) return st;
    if (!any_type(in_type)) return PVMVMD_E_ARG;
    if (q_dev && Hq < 1) return PVMVMD_E_SHAPE;
    if (kv.T == 0) return PVMVMD_OK;
    if (!k_dev || !v_dev || (q_dev && !q_out_dev)) return PVMVMD_E_ARG;
    RopeJob j{};
    if (rope) {
        j.turns = rope->turns_dev;
        j.rot = rope->rot;
        j.interleaved = rope->interleaved != 0;
        j.magnitude = rope->magnitude;
    }
    j.pos = pos_dev;
    if (q_dev) j.part[0] = RopePart{q_dev, q_out_dev, q_token, q_head, q_out_token, q_out_head, Hq};
    j.part[1] = RopePart{k_dev, nullptr, k_token, k_head, 0, 0, kv.heads};
    j.part[2] = RopePart{v_dev, nullptr, v_token, v_head, 0, 0, kv.heads};
    j.T = kv.T;
    j.dim = kv.dim;
    j.in_type = in_type;
    j.out_type = pool->type;
    j.scale = scale;
    j.cached = true;
    PV_CUDA(launch_rope(j, &kv, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}

int pvmvmd_paged_attention(const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch, int Hq, const void *q_dev,
                           int64_t q_token, int64_t q_head, float scale, int causal, int window, int accumulate,
                           void *out_dev, int64_t out_token, int64_t out_head, float *lse_dev, void *stream) {
    using namespace pv;
    KvView kv;
    int st = view(pool, batch, kv);
    if (!st) st = check_new(batch);
    if (st) return st;
    if (Hq < 1 || Hq % kv.heads || window < 0) return PVMVMD_E_SHAPE;
    if (accumulate && !kv.mass) return PVMVMD_E_ARG;
    if (kv.T == 0) return PVMVMD_OK;
    if (!q_dev || !out_dev || !aligned16(q_dev) || !aligned16(out_dev) || !rows16(q_token, q_head) ||
        !rows16(out_token, out_head))
        return PVMVMD_E_ARG;
    if ((int64_t)kv.T * Hq > INT_MAX) return PVMVMD_E_SHAPE;
    AttendJob j{};
    j.q = q_dev;
    j.out = out_dev;
    j.lse = lse_dev;
    j.q_token = 2 * q_token;
    j.q_head = 2 * q_head;
    j.o_token = 2 * out_token;
    j.o_head = 2 * out_head;
    j.Hq = Hq;
    j.window = window;
    j.type = pool->type;
    j.max_new = kv.max_new;
    j.scale = scale;
    j.causal = causal != 0;
    j.accumulate = accumulate != 0;
    const StreamTurn turn(static_cast<cudaStream_t>(stream));
    if (!turn) return PVMVMD_E_NOMEM;
    PV_CUDA(launch_attention(j, kv, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}

int pvmvmd_kv_evict(const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch, int budget, int recent,
                    const int32_t *new_table_dev, int64_t new_table_stride, int new_max_pages, int32_t *new_lens_dev,
                    void *stream) {
    using namespace pv;
    KvView kv;
    const int st = view(pool, batch, kv);
    if (st) return st;
    if (!new_table_dev || !new_lens_dev || !kv.mass) return PVMVMD_E_ARG;
    if (budget < 1 || recent < 0 || new_max_pages < 1) return PVMVMD_E_SHAPE;
    const int64_t room = (int64_t)new_max_pages * pool->page_size;
    if (room < budget && room < (int64_t)kv.max_pages * pool->page_size) return PVMVMD_E_SHAPE;
    const EvictJob j{budget, recent, new_table_dev, new_table_stride, new_lens_dev};
    const StreamTurn turn(static_cast<cudaStream_t>(stream));
    if (!turn) return PVMVMD_E_NOMEM;
    PV_CUDA(launch_evict(j, kv, static_cast<cudaStream_t>(stream)));
    return PVMVMD_OK;
}
