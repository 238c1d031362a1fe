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

// 16 bytes of Out and as many values of In.
template <typename T, int N>
struct __align__(sizeof(T) * N) Vec {
    T v[N];
};
constexpr int kGroup = 8;  // values that a thread takes at a time

template <typename T>
struct Raw {
    static constexpr int kN = 16 / sizeof(T);
    Vec<T, kN> u[kGroup / kN];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < kGroup / kN; ++i) u[i] = *reinterpret_cast<const Vec<T, kN> *>(p + i * kN);
    }
    __device__ __forceinline__ void get(float scale, float (&x)[kGroup]) const {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) x[i] = to_f32(u[i / kN].v[i % kN]) * scale;
    }
};
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

// 16 bytes at a time, for rows on 16-byte boundaries.  A thread owns 8 values of a
// token, or the two groups of 8 that make pairs, and takes them through several
// heads, so that it forms their angles once: without that the sines bound it (a chunk
// of 6001 tokens, 80 heads of 128, took 283 us with them formed for every head).
// kHalves: pairs are half a rotation apart, not side by side.
template <typename In, typename Out, bool kHalves>
__global__ void __launch_bounds__(kRopeThreads) k_rope_rows(const __grid_constant__ RopeArgs a, int units, int split,
                                                           int per) {
    const RopeJob &j = a.j;
    const int64_t id = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    const int u = (int)(id % units);
    const int64_t ts = id / units;
    const int t = (int)(ts / split), h0 = (int)(ts % split) * per, h1 = min(a.heads, h0 + per);
    if (ts / split >= j.T) return;
    int b = 0, page = 0, slot = 0, idx = 0;
    bool placed = false;
    if (j.cached) {
        b = a.kv.seq(t);
        idx = a.kv.len(b) - a.kv.news(b) + t - a.kv.first(b);
        placed = idx >= 0 && a.kv.place(b, idx, page, slot);
    }
    const int turning = kHalves ? j.rot / (2 * kGroup) : j.rot / kGroup;  // units that are rotated
    const bool mine = u < turning;
    const int d0 = mine || !kHalves ? u * kGroup : j.rot + (u - turning) * kGroup, d1 = d0 + j.rot / 2;
    float c[kGroup], s[kGroup];
    if (mine && h0 < j.part[0].heads + j.part[1].heads) {
        const int pos = j.pos ? j.pos[t] : idx;
#pragma unroll
        for (int e = 0; e < (kHalves ? kGroup : kGroup / 2); ++e) sincos_at(j, kHalves ? d0 + e : d0 / 2 + e, pos, c[e], s[e]);
    }
    // some heads' loads in flight before the first is stored (out may be x itself)
    constexpr int kAhead = sizeof(In) == 2 ? 4 : 2;
    for (int hb = h0; hb < h1; hb += kAhead) {
        Raw<In> raw0[kAhead], raw1[kAhead];
        Out *to[kAhead];
        bool turn[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int h = hb + i;
            const In *src;
            to[i] = nullptr;
            if (h >= h1) continue;
            head_rows(a, t, h, b, page, slot, placed, src, to[i], turn[i]);
            if (j.cached && a.kv.mass && placed && u == 0 && h >= j.part[0].heads &&
                h < j.part[0].heads + j.part[1].heads)
                *a.kv.mass_at(page, slot, h - j.part[0].heads) = 0.0f;
            if (!to[i]) continue;
            raw0[i].load(src + d0);
            if (kHalves && mine) raw1[i].load(src + d1);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (!to[i]) continue;
            float x[kGroup], y[kGroup];
            raw0[i].get(j.scale, x);
            if (kHalves && mine) {
                raw1[i].get(j.scale, y);
                if (turn[i])
#pragma unroll
                    for (int e = 0; e < kGroup; ++e) {
                        const float p = x[e], q = y[e];
                        x[e] = p * c[e] - q * s[e];
                        y[e] = p * s[e] + q * c[e];
                    }
                store8(to[i] + d1, y);
            } else if (!kHalves && mine && turn[i]) {
#pragma unroll
                for (int e = 0; e < kGroup / 2; ++e) {
                    const float p = x[2 * e], q = x[2 * e + 1];
                    x[2 * e] = p * c[e] - q * s[e];
                    x[2 * e + 1] = p * s[e] + q * c[e];
                }
            }
            store8(to[i] + d0, x);
        }
    }
}

// Rows on 16-byte boundaries, in whole groups.
template <typename In, typename Out>
bool rows_ok(const RopeArgs &a) {
    const RopeJob &j = a.j;
    if (j.dim % kGroup || j.rot % (j.interleaved ? kGroup : 2 * kGroup)) return false;
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
        // heads a thread: few while that leaves SMs without threads, at most 16
        const int64_t threads = (int64_t)j.T * units * a.heads;
        const int per = (int)std::max<int64_t>(1, std::min<int64_t>(16, threads / (152 * 1024)));
        const int split = (a.heads + per - 1) / per;
        const unsigned grid = (unsigned)(((int64_t)j.T * units * split + kRopeThreads - 1) / kRopeThreads);
        if (j.interleaved)
            k_rope_rows<In, Out, false><<<grid, kRopeThreads, 0, s>>>(a, units, split, per);
        else
            k_rope_rows<In, Out, true><<<grid, kRopeThreads, 0, s>>>(a, units, split, per);
        return counted_launch(cudaGetLastError());
    }
    const int64_t n = (int64_t)j.T * a.heads * (j.rot / 2 + j.dim - j.rot);
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
