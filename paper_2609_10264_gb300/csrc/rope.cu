// Rotary positions (pvmvmd_rope) and the append of new tokens to a paged cache
// (pvmvmd_kv_append): one kernel over the heads of a token, rotated or copied, to
// rows of a tensor or of a page.
//
// Angles.  A frequency is a fraction of a turn per position in units of 2^-64, so
// position * frequency modulo 2^64 is the angle modulo whole turns, exactly, at
// any position; its upper 32 bits, read as signed, go to sincospi with an error of
// 2^-24 of the angle.  (In 32-bit floating point the angle alone is 2^-9 off at
// position 30000.)
#include <algorithm>

#include "attention.h"
#include "kv.cuh"

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

// Source and destination of head h (of all three parts) of token t; null where
// there is nothing to write.
template <typename In, typename Out>
__device__ __forceinline__ void head_rows(const RopeArgs &a, int t, int h, int b, int page, int slot, bool placed,
                                          const In *&src, Out *&dst, bool &rotate) {
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
    if (placed)
        dst = reinterpret_cast<Out *>(v ? a.kv.V + page * a.kv.v_page + slot * a.kv.v_slot + h * a.kv.v_head
                                        : a.kv.K + page * a.kv.k_page + slot * a.kv.k_slot + h * a.kv.k_head);
}

// One thread per (token, head, value pair or copied value): any strides.
template <typename In, typename Out>
__global__ void __launch_bounds__(kRopeThreads) k_rope_any(const __grid_constant__ RopeArgs a) {
    const RopeJob &j = a.j;
    const int half = j.rot / 2, units = half + j.dim - j.rot;
    const int64_t id = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    const int u = (int)(id % units);
    const int64_t th = id / units;
    const int h = (int)(th % a.heads);
    if (th / a.heads >= j.T) return;
    const int t = (int)(th / a.heads);
    int b = 0, page = 0, slot = 0, idx = 0;
    bool placed = false;
    if (j.cached) {
        b = a.kv.seq(t);
        idx = a.kv.len(b) - a.kv.news(b) + t - a.kv.first(b);
        placed = idx >= 0 && a.kv.place(b, idx, page, slot);
    }
    const In *src;
    Out *dst;
    bool rotate;
    head_rows(a, t, h, b, page, slot, placed, src, dst, rotate);
    if (j.cached && a.kv.mass && placed && u == 0 && h >= j.part[0].heads && h < j.part[0].heads + j.part[1].heads)
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

template <typename In, typename Out>
cudaError_t rope_launch(const RopeArgs &a, cudaStream_t s) {
    const int64_t n = (int64_t)a.j.T * a.heads * (a.j.rot / 2 + a.j.dim - a.j.rot);
    k_rope_any<In, Out><<<(unsigned)((n + kRopeThreads - 1) / kRopeThreads), kRopeThreads, 0, s>>>(a);
    return counted_launch(cudaGetLastError());
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
