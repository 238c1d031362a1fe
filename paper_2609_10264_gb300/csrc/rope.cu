// Rotary positions (pvmvmd_rope) and the append of new tokens to a paged cache
// (pvmvmd_kv_append): one kernel over the heads of a token, rotated or copied, to
// rows of a tensor or of a page.
//
// Angles.  A frequency is a fraction of a turn per position in units of 2^-64, so
// position * frequency modulo 2^64 is the angle modulo whole turns, exactly, at
// any position; its upper 32 bits, read as signed, go to sincospi with an error of
// 2^-24 of the angle.  (In 32-bit floating point the angle alone is 2^-9 off at
// position 30000.)
//
// Bound by memory: 4097 tokens of 32 heads of 96 in 32 bits 18 us (5.5 TB/s), 6001
// tokens of 64 + 8 + 8 heads of 128 into a cache 46 us (5.3 TB/s).
#include <algorithm>

#include "attention.cuh"

namespace pv {
namespace {

constexpr int kRopeThreads = 128;

struct RopeArgs {
    RopeJob j;
    KvView kv;  // where heads go to the cache
    int heads;  // of all three parts
};

__device__ __forceinline__ void sincos_at(const RopeJob &j, int pair, int pos, float &c, float &s) {
    const uint64_t turn = (uint64_t)(int64_t)pos * j.turns[pair];
    const float half_turns = (float)(int32_t)(turn >> 32) * 4.656612873077393e-10f;  // 2^-31
    sincospif(half_turns, &s, &c);
    c *= j.magnitude;
    s *= j.magnitude;
}

// Source and destination of head h (of all three parts) of token t, which goes to
// the slot of the page; null where there is nothing to write (page < 0).
template <typename In, typename Out>
__device__ __forceinline__ void head_rows(const RopeArgs &a, int t, int h, int page, int slot, const In *&src, Out *&dst,
                                          bool &rotate) {
    const RopeJob &j = a.j;
    if (h < j.part[0].heads) {
        src = static_cast<const In *>(j.part[0].src) + t * j.part[0].src_token + h * j.part[0].src_head;
        dst = static_cast<Out *>(j.part[0].dst) + t * j.part[0].dst_token + h * j.part[0].dst_head;
        rotate = j.rot > 0;
        return;
    }
    h -= j.part[0].heads;
    const bool v = h >= j.part[1].heads;
    if (v) h -= j.part[1].heads;
    const RopePart &p = j.part[1 + v];
    src = static_cast<const In *>(p.src) + t * p.src_token + h * p.src_head;
    rotate = !v && j.rot > 0;
    dst = nullptr;
    if (page >= 0)
        dst = reinterpret_cast<Out *>(v ? a.kv.V + page * a.kv.v_page + slot * a.kv.v_slot + h * a.kv.v_head
                                        : a.kv.K + page * a.kv.k_page + slot * a.kv.k_slot + h * a.kv.k_head);
}

// One thread per (token, head, value pair or copied value): any strides, and rotations
// that are not whole groups of 8.  Bound by the sines, which every head forms for itself:
// 6001 tokens of 80 heads of 80, of which 40 are rotated in halves, 232 us where their
// bytes take 23; of 128, of which 120 are, 263 (k_rope_rows takes all 128 in 50).
template <typename In, typename Out>
__global__ void __launch_bounds__(kRopeThreads) k_rope_any(const __grid_constant__ RopeArgs a) {
    follow();
    const RopeJob &j = a.j;
    const int half = j.rot / 2, units = half + j.dim - j.rot;
    const int64_t id = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    const int u = (int)(id % units);
    const int64_t th = id / units;
    const int h = (int)(th % a.heads);
    if (th / a.heads >= j.T) return;
    const int t = (int)(th / a.heads);
    int b = 0, page = -1, slot = 0, idx = 0;
    if (j.cached) {
        b = a.kv.seq(t);
        idx = a.kv.index(b, t);
        if (idx < 0 || !a.kv.place(b, idx, page, slot)) page = -1;
    }
    const In *src;
    Out *dst;
    bool rotate;
    head_rows(a, t, h, page, slot, src, dst, rotate);
    if (j.cached && a.kv.mass && page >= 0 && u == 0 && h >= j.part[0].heads && h < j.part[0].heads + j.part[1].heads)
        *a.kv.mass_at(page, slot, h - j.part[0].heads) = 0.0f;
    if (!dst) return;
    if (u >= half) {
        const int d = j.rot + u - half;
        dst[d] = from_f32<Out>(to_f32(src[d]) * j.scale);
        return;
    }
    const int d0 = j.interleaved ? 2 * u : u, d1 = j.interleaved ? 2 * u + 1 : u + half;
    const float x = to_f32(src[d0]) * j.scale, y = to_f32(src[d1]) * j.scale;
    float c = 1.0f, s = 0.0f;
    if (rotate) {
        sincos_at(j, u, j.pos ? j.pos[t] : idx, c, s);
        dst[d0] = from_f32<Out>(x * c - y * s);
        dst[d1] = from_f32<Out>(x * s + y * c);
    } else {
        dst[d0] = from_f32<Out>(x);
        dst[d1] = from_f32<Out>(y);
    }
}

// 16 bytes of Out and as many values of In.
template <typename T, int N>
struct __align__(sizeof(T) * N) Vec {
    T v[N];
};
constexpr int kGroup = 8;  // values that a thread takes at a time

template <typename T>
__device__ __forceinline__ void load8(const T *p, float scale, float (&x)[kGroup]) {
    constexpr int kN = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kGroup; i += kN) {
        const Vec<T, kN> u = *reinterpret_cast<const Vec<T, kN> *>(p + i);
#pragma unroll
        for (int e = 0; e < kN; ++e) x[i + e] = to_f32(u.v[e]) * scale;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&x)[kGroup]) {
    constexpr int kN = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < kGroup; i += kN) {
        Vec<T, kN> u;
#pragma unroll
        for (int e = 0; e < kN; ++e) u.v[e] = from_f32<T>(x[i + e]);
        *reinterpret_cast<Vec<T, kN> *>(p + i) = u;
    }
}

// 16 bytes at a time, for rows on 16-byte boundaries.  A CTA takes some tokens
// through some heads: it forms the tokens' sines and places once, in shared memory,
// and then every thread 8 values of a head, or the two groups of 8 that make pairs
// (more of them at a time cost registers, and with them warps in flight).  Bound by
// the copy: 6001 tokens of 80 heads of 128 took 283 us with sines formed for every
// head, 95 with a token's formed by each thread.
// kHalves: pairs are half a rotation apart, not side by side.
constexpr int kRowThreads = 256;
constexpr int kMostTokens = 8;
constexpr int kMostSines = 1024;  // tokens x pairs of a CTA
struct RowPlan {
    int tokens, heads;  // of a CTA
    FastDiv units, per; // threads per head; heads
};
template <typename In, typename Out, bool kHalves>
__global__ void __launch_bounds__(kRowThreads, 8) k_rope_rows(const __grid_constant__ RopeArgs a,
                                                          const __grid_constant__ RowPlan plan) {
    follow();
    const RopeJob &j = a.j;
    __shared__ __align__(16) float s_cos[kMostSines], s_sin[kMostSines];
    __shared__ int s_page[kMostTokens], s_slot[kMostTokens];  // page -1: nowhere
    const int tid = threadIdx.x, half = j.rot / 2;
    const int t0 = blockIdx.x * plan.tokens, nt = min(plan.tokens, j.T - t0);
    const int h0 = blockIdx.y * plan.heads, nh = min(plan.heads, a.heads - h0);
    const int turned = j.part[0].heads + j.part[1].heads;  // heads that are rotated
    auto index_of = [&](int t, int &b) {  // the token's cache index
        b = a.kv.seq(t);
        return a.kv.index(b, t);
    };
    if (j.cached && tid < nt) {
        int b, page, slot;
        const int idx = index_of(t0 + tid, b);
        const bool placed = idx >= 0 && a.kv.place(b, idx, page, slot);
        s_page[tid] = placed ? page : -1;
        s_slot[tid] = placed ? slot : 0;
    }
    if (h0 < turned)
        for (int i = tid; i < nt * half; i += kRowThreads) {
            const int t = i / half, e = i - t * half;
            int b;
            const int pos = j.pos ? j.pos[t0 + t] : index_of(t0 + t, b);
            sincos_at(j, e, pos, s_cos[i], s_sin[i]);
        }
    __syncthreads();
    const int turning = kHalves ? half / kGroup : j.rot / kGroup;  // units that are rotated
    const int units = (int)plan.units.d, all = nt * nh * units;
    for (int i = tid; i < all; i += kRowThreads) {
        uint32_t row, u, t, h;
        plan.units.divmod((uint32_t)i, row, u);
        plan.per.divmod(row, t, h);
        h += h0;
        const int page = j.cached ? s_page[t] : -1, slot = j.cached ? s_slot[t] : 0;
        const In *src;
        Out *dst;
        bool rotate;
        head_rows(a, t0 + (int)t, (int)h, page, slot, src, dst, rotate);
        if (j.cached && a.kv.mass && page >= 0 && u == 0 && (int)h >= j.part[0].heads && (int)h < turned)
            *a.kv.mass_at(page, slot, (int)h - j.part[0].heads) = 0.0f;
        if (!dst) continue;
        const bool mine = (int)u < turning;
        const int d0 = mine || !kHalves ? (int)u * kGroup : j.rot + ((int)u - turning) * kGroup;
        float x[kGroup], y[kGroup];
        load8(src + d0, j.scale, x);
        if (kHalves && mine) load8(src + d0 + half, j.scale, y);
        if (mine && rotate) {
            const int at = (int)t * half + (kHalves ? d0 : d0 / 2);
#pragma unroll
            for (int e = 0; e < (kHalves ? kGroup : kGroup / 2); ++e) {
                float &p = kHalves ? x[e] : x[2 * e], &q = kHalves ? y[e] : x[2 * e + 1];
                const float c = s_cos[at + e], s = s_sin[at + e], px = p, qx = q;
                p = px * c - qx * s;
                q = px * s + qx * c;
            }
        }
        if (kHalves && mine) store8(dst + d0 + half, y);
        store8(dst + d0, x);
    }
}

// Rows on 16-byte boundaries, in whole groups.
template <typename In, typename Out>
bool rows_ok(const RopeArgs &a) {
    const RopeJob &j = a.j;
    if (j.dim % kGroup || j.rot % (j.interleaved ? kGroup : 2 * kGroup) || j.rot / 2 > kMostSines) return false;
    for (const RopePart &p : j.part) {
        if (!p.heads) continue;
        if (reinterpret_cast<uintptr_t>(p.src) % 16 || p.src_token * sizeof(In) % 16 || p.src_head * sizeof(In) % 16)
            return false;
        if (p.dst && (reinterpret_cast<uintptr_t>(p.dst) % 16 || p.dst_token * sizeof(Out) % 16 ||
                      p.dst_head * sizeof(Out) % 16))
            return false;
    }
    return true;
}

template <typename In, typename Out>
cudaError_t rope_launch(const RopeArgs &a, cudaStream_t s) {
    const RopeJob &j = a.j;
    if (rows_ok<In, Out>(a)) {
        const int units = j.interleaved ? j.dim / kGroup : j.rot / (2 * kGroup) + (j.dim - j.rot) / kGroup;
        // Heads a CTA: all, or as many as four turns of its threads take where the
        // tokens alone would leave SMs without one.  Tokens a CTA: up to six turns, but more
        // than one turn only where twelve CTAs an SM are left (eight run at a time, so that
        // fewer leave a long tail: 4097 tokens of 32 heads of 96 in 32 bits with 1 token a
        // CTA 18.9 us, 2 18.2, 3 21.0, 4 22.8, 5 23.5).
        const int turn = std::max(1, kRowThreads / units), sms = 152;
        RowPlan plan;
        plan.heads = j.T >= 4 * sms ? a.heads : std::min(a.heads, j.T >= sms ? 4 * turn : turn);
        plan.heads = std::max(plan.heads, a.heads / 65535 + 1);  // a grid's second dimension ends there
        plan.tokens = std::max(1, std::min({kMostTokens, kMostSines / std::max(1, j.rot / 2), 6 * turn / plan.heads,
                                            j.T / (4 * sms), std::max(j.T / (12 * sms), turn / plan.heads)}));
        plan.units = FastDiv((uint32_t)units);
        plan.per = FastDiv((uint32_t)plan.heads);
        const dim3 grid((unsigned)((j.T + plan.tokens - 1) / plan.tokens),
                        (unsigned)((a.heads + plan.heads - 1) / plan.heads));
        return launch_dependent(j.interleaved ? k_rope_rows<In, Out, false> : k_rope_rows<In, Out, true>, grid, kRowThreads,
                                0, s, a, plan);
    }
    const int64_t n = (int64_t)j.T * a.heads * (j.rot / 2 + j.dim - j.rot);
    return launch_dependent(k_rope_any<In, Out>, dim3((unsigned)((n + kRopeThreads - 1) / kRopeThreads)), kRopeThreads, 0,
                            s, a);
}
template <typename In>
cudaError_t rope_out(const RopeArgs &a, cudaStream_t s) {
    switch (a.j.out_type) {
        case PVMVMD_BF16: return rope_launch<In, __nv_bfloat16>(a, s);
        case PVMVMD_F16: return rope_launch<In, __half>(a, s);
        default: return rope_launch<In, float>(a, s);
    }
}

}  // namespace

cudaError_t launch_rope(const RopeJob &j, const KvView *kv, cudaStream_t s) {
    RopeArgs a;
    a.j = j;
    if (kv) a.kv = *kv;
    a.heads = j.part[0].heads + j.part[1].heads + j.part[2].heads;
    switch (j.in_type) {
        case PVMVMD_BF16: return rope_out<__nv_bfloat16>(a, s);
        case PVMVMD_F16: return rope_out<__half>(a, s);
        case PVMVMD_F32: return rope_out<float>(a, s);
        default: return rope_out<uint32_t>(a, s);
    }
}

}  // namespace pv
