// Attention of sequences with few new rows (new tokens x query heads of a key head):
// single generated tokens above all.  Bound by the reading of K and V: 131071 keys of 8
// heads of 128 89-91 us a call (6.0 TB/s); 64 sequences of up to 8192 with their weights
// 172 us (6.7 TB/s with the scores written), and 28 to finish.
//
// Work.  The keys of a (sequence, key head) come in tiles of 64 or 128.  All tiles of all
// of them, one after the other, are dealt out evenly to the CTAs, whatever the
// sequences' lengths: CTA c of C takes tiles [N c / C, N (c + 1) / C).  A sequence
// that one CTA has whole is finished there; parts go to scratch as (maximum, sum,
// unnormalised output), and k_few_finish puts them together in order.
//
// A warp takes a quarter of a tile's keys through its own ring of asynchronous copies
// and keeps its own running maximum and sum, so that nothing but the end of a
// sequence waits for another warp.  Both products are m16n8k16 MMAs with the rows
// padded to 16 (tcgen05 would pad them to 128, and its operands would all pass
// through one barrier per tile).  P is split into two 16-bit parts, which leaves its
// rounding at 2^-17: the MMAs are not what bounds this.
#include <algorithm>

#include "attention.h"
#include "attention.cuh"

namespace pv {
namespace {

constexpr int kRows = 16;                 // rows per tile of them, of one MMA
constexpr float kHeadroom = 8.0f;         // log2 of the largest P

struct FewArgs {
    AttendJob j;
    KvView kv;
    float *part;     // [2 C][kRows][DP] unnormalised partial outputs
    float2 *stat;    // [2 C][kRows] their maximum and sum
    int64_t *before; // [B + 1] work before each sequence, and all of it
    float2 *norm;    // [T][Hq] maximum and 1 / sum, where mass is accumulated
    float *scores;   // [B][heads][max tiles x tile][rows] where mass is accumulated (see seen_keys)
    int score_rows, max_tiles;  // (rows a multiple of 4)
    float scale2;    // scale x log2(e)
    int G, C;
    int tile_log;    // keys per tile
    unsigned finishers;  // CTAs of k_few_finish for a key head and tile of rows
    bool whole;      // a CTA takes all keys of a row tile
};

// DP: the head's values in whole MMAs of the columns that are built (64, 96, 128).
// W: warps, four of each of two CTAs of an SM; eight of one where a CTA takes all keys of
// a row tile and there are no more of these than SMs (8 heads, 200 keys: 5.5 us a call,
// with four 6.7; 20 such sequences 9.8 and 7.1).
template <int DP, int W>
struct Few {
    static constexpr int kThreads = 32 * W;
    // Keys per warp and step, and steps of the ring: what two CTAs of an SM have room for.
    // 32 keys take less than two steps of 16 (57 ragged sequences of up to 3481 keys, 8 heads
    // of 64 in pages of 16, 64, 100 and 1: 47, 45, 49 and 50 us a call where 16 keys in a
    // ring of six steps took 50, 47, 54 and 59; heads of 96: 68 to 72 where 69 to 78).
    static constexpr int kSub = DP == 128 ? 16 : 32;
    static constexpr int kStages = DP == 96 ? 2 : 3;
    static constexpr int kTile = W * kSub;  // keys per tile
    static_assert(kTile <= kFewMostTile);
    // bytes of a row; chunks of 16 are swizzled, or rows of 13 chunks where 12 are used:
    // either way 8 rows' chunks lie in different banks
    static constexpr int kRow = DP == 96 ? 208 : 2 * DP;
    static __device__ __forceinline__ int at(int r, int ch) { return r * kRow + ((DP == 96 ? ch : ch ^ (r & 7)) << 4); }
    static constexpr int kHalf = kSub * kRow;
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kRing = W * kStages * kStage;
    static constexpr int kSmem = kRing + kRows * kRow;
    static constexpr int kChunks = DP / 8;
    static constexpr int kWave = 32 / kChunks;  // rows that a warp copies at a time
    static constexpr int kDeep = DP == 96 ? 3 : 4;  // MMAs' operands that are read ahead
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (sizeof(T) == 2 && __is_same(T, __half))
        asm(
            "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm(
            "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two values as a 16-bit pair and the pair of what that leaves
template <typename T>
__device__ __forceinline__ void split(float x, float y, uint32_t &hi, uint32_t &lo) {
    const T a = from_f32<T>(x), b = from_f32<T>(y);
    hi = pack(x, y, T{});
    lo = pack(x - to_f32(a), y - to_f32(b), T{});
}
// ---------------------------------------------------------------- work
// One sequence's share: of each key head and tile of kRows rows, `tiles` tiles of keys
// from key `first` on, dealt out in `units`: the tiles, behind kSetUp empty units for
// what a CTA does before and after them (57 sequences of 70 to 3481 keys, 8 heads of 64:
// 45 us a call where 58 without, when one CTA had several short ones).
constexpr int kSetUp = 3;
struct Share {
    int len, n, row0;  // cached and new tokens, the first of these
    int rows, rts, first, tiles, units;
    int64_t work;  // units of all
};
__device__ __forceinline__ Share share(const FewArgs &a, int b) {
    Share s;
    s.row0 = a.kv.first(b);
    s.n = a.kv.news(b);
    s.len = a.kv.len(b);
    s.rows = s.n * a.G;
    s.rts = (s.rows + kRows - 1) / kRows;
    const int at = s.len - s.n;  // of the first new token
    s.first = a.j.window > 0 && at >= a.j.window ? (at - a.j.window + 1) >> a.tile_log << a.tile_log : 0;
    s.tiles = max(1, (s.len - s.first + (1 << a.tile_log) - 1) >> a.tile_log);
    s.units = a.whole ? 1 : kSetUp + s.tiles;
    s.work = s.rows <= 0 || s.rows > a.j.few_rows ? 0 : (int64_t)s.units * a.kv.heads * s.rts;
    return s;
}
// The first position of CTA c of C <= N.
__device__ __forceinline__ int64_t cut(int64_t N, int c, int64_t C) { return N == C ? c : N * c / C; }
// The CTA that takes position p of N, among C <= N.
__device__ __forceinline__ int owner(int64_t p, int64_t N, int64_t C) { return (int)(((p + 1) * C - 1) / N); }

// Four values of row r of a sequence and key head, from value d on.
template <typename T>
__device__ __forceinline__ void put_row(const FewArgs &a, int row0, int hk, int r, int d, float4 v, float inv) {
    if (d >= a.kv.dim) return;
    const int t = row0 + r / a.G, h = hk * a.G + r % a.G;
    *reinterpret_cast<uint2 *>(static_cast<char *>(a.j.out) + t * a.j.o_token + h * a.j.o_head + 2 * d) =
        make_uint2(pack(v.x * inv, v.y * inv, T{}), pack(v.z * inv, v.w * inv, T{}));
}

// ---------------------------------------------------------------- main kernel
template <typename T, int DP, int W>
__global__ void __launch_bounds__(Few<DP, W>::kThreads, 8 / W) k_few(const __grid_constant__ FewArgs a) {
    using F = Few<DP, W>;
    constexpr int kSub = F::kSub, kTile = F::kTile;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float2 s_stat[W][kRows];
    const AttendJob &j = a.j;
    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane & 3, grp = lane >> 2;
    follow();
    const Found f = find<F::kThreads>(
        kv.B, [&](int b) { return share(a, b).work; },
        [&](int64_t total) {
            const int64_t C = min((int64_t)a.C, total);
            return (int64_t)blockIdx.x < C ? cut(total, blockIdx.x, C) : -1;
        },
        blockIdx.x == 0 ? a.before : nullptr);
    const int64_t C = min((int64_t)a.C, f.total);
    if ((int64_t)blockIdx.x >= C) return;
    const int64_t p1 = cut(f.total, blockIdx.x + 1, C);
    int64_t p = cut(f.total, blockIdx.x, C), done = f.before;
    int b = f.b;
    Share sh = share(a, b);
    const uint32_t ring = smem_addr(smem) + warp * F::kStages * F::kStage, qs = smem_addr(smem) + F::kRing;
    const bool one_page = kv.ps.d % 16 == 0;  // for 16 keys
    const int chunks = kv.dim / 8;

    while (p < p1) {
        while (p >= done + sh.work) {
            done += sh.work;
            sh = share(a, ++b);
        }
        const int64_t in = p - done;
        const int item = a.whole             ? (int)in
                         : sh.work >> 32 == 0 ? (int)((uint32_t)in / (uint32_t)sh.units)
                                              : (int)(in / sh.units);
        const int u0 = (int)(in - (int64_t)item * sh.units);
        const int units = a.whole ? 1 : (int)min((int64_t)(sh.units - u0), p1 - p);
        p += units;
        const int t0 = a.whole ? 0 : max(0, u0 - kSetUp), nt = a.whole ? sh.tiles : u0 + units - kSetUp - t0;
        if (nt <= 0) continue;
        const int hk = item / sh.rts, r0 = item % sh.rts * kRows, rows = min(kRows, sh.rows - r0);
        const int len = sh.len, n = sh.n, row0 = sh.row0;
        // ---- this warp's step i: keys from key0(i) on
        auto key0 = [&](int i) { return sh.first + (t0 + i) * kTile + warp * kSub; };
        int pages[F::kStages];  // of the steps to be loaded next, a lane a key
        auto fetch_page = [&](int i) {
            const int k = key0(i) + (lane & (kSub - 1));
#pragma unroll
            for (int s = 0; s + 1 < F::kStages; ++s) pages[s] = pages[s + 1];
            pages[F::kStages - 1] = -1;
            if (i < nt && k < len) {
                uint32_t q, r;
                kv.ps.divmod((uint32_t)k, q, r);
                pages[F::kStages - 1] = kv.table[b * kv.table_stride + q];
            }
        };
        unsigned seen[F::kStages] = {};  // of the steps loaded last: the keys that are there
        auto load = [&](int i) {  // step i's copies (its pages have been fetched)
            unsigned there = 0;
            const int page = pages[0];
            if (i < nt) {
                const int k0 = key0(i), ch = lane % F::kChunks, sub = lane / F::kChunks;
                const bool mine = page >= 0 && page < kv.pages && k0 + (lane & (kSub - 1)) < len;
                there = __ballot_sync(kFull, mine);
                const uint32_t st = ring + (i % F::kStages) * F::kStage;
                const char *ks = nullptr, *vs = nullptr;
                // a row's chunks by neighbouring lanes; rows of K, and of V behind them
#pragma unroll
                for (int u = 0; u < kSub / F::kWave; ++u) {
                    const int r = u * F::kWave + sub;
                    if (!one_page || u % (16 / F::kWave) == 0) {
                        const int pg = __shfl_sync(kFull, page, r);
                        uint32_t q, o;
                        kv.ps.divmod((uint32_t)(k0 + r), q, o);
                        ks = kv.K + pg * kv.k_page + o * kv.k_slot + hk * kv.k_head + ch * 16;
                        vs = kv.V + pg * kv.v_page + o * kv.v_slot + hk * kv.v_head + ch * 16;
                    }
                    const bool real = (there >> r & 1) && ch < chunks;
                    if (sub < F::kWave) {
                        copy16(st + F::at(r, ch), real ? ks : kv.K, real);
                        copy16(st + F::kHalf + F::at(r, ch), real ? vs : kv.V, real);
                    }
                    ks += F::kWave * kv.k_slot;
                    vs += F::kWave * kv.v_slot;
                }
            }
#pragma unroll
            for (int s = 0; s + 1 < F::kStages; ++s) seen[s] = seen[s + 1];
            seen[F::kStages - 1] = there;
            copy_commit();
        };
#pragma unroll
        for (int i = 0; i < F::kStages; ++i) fetch_page(i);
        // rows of Q, zero beyond the real ones
        for (int id = tid; id < kRows * F::kChunks; id += F::kThreads) {
            const int r = id / F::kChunks, ch = id % F::kChunks;
            const bool real = r < rows && ch < chunks;
            const char *src = static_cast<const char *>(j.q);
            if (real)
                src += (int64_t)(row0 + (r0 + r) / a.G) * j.q_token + (int64_t)(hk * a.G + (r0 + r) % a.G) * j.q_head + ch * 16;
            copy16(qs + F::at(r, ch), src, real);
        }
        copy_commit();
#pragma unroll
        for (int i = 0; i < F::kStages - 1; ++i) {
            load(i);
            fetch_page(i + F::kStages);
        }
        copy_wait<F::kStages - 1>();
        __syncthreads();
        uint32_t qf[DP / 16][4];
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            const int r = lane & 15, ch = 2 * k + (lane >> 4);
            ldsm4(qs + F::at(r, ch), qf[k]);
        }
        // keys that rows grp and grp + 8 see
        int lo[2], hi[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = grp + 8 * h, at = len - n + (r0 + r) / a.G;
            hi[h] = r < rows && j.causal ? min(len, at + 1) : len;
            lo[h] = r < rows && j.window > 0 && at >= j.window ? at - j.window + 1 : 0;
        }
        // keys that all of them see
        const int all_lo = __reduce_max_sync(kFull, max(lo[0], lo[1]));
        const int all_hi = __reduce_min_sync(kFull, min(hi[0], hi[1]));
        float o[DP / 8][4] = {}, m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
        for (int i = 0; i < nt; ++i) {
            copy_wait<F::kStages - 2>();
            __syncwarp();
            load(i + F::kStages - 1);
            fetch_page(i + 2 * F::kStages - 1);
            const uint32_t st = ring + (i % F::kStages) * F::kStage;
            const int k0 = key0(i);
            if (k0 >= len) continue;  // the same for the whole warp
            const unsigned there = seen[0];
            constexpr int kEights = kSub / 8;
            // two sums of 8 keys where these are few, so that the MMAs wait less for one another
            constexpr int kSums = kEights == 2 ? 2 : 1;
            float s[kEights][4], sums[kSums][kEights][4] = {};
#pragma unroll
            for (int k = 0; k < DP / 16; k += F::kDeep) {
#pragma unroll
                for (int t = 0; t < kEights; t += 2) {
                    uint32_t kf[F::kDeep][4];
                    const int r = 8 * t + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                    for (int u = 0; u < F::kDeep; ++u) ldsm4(st + F::at(r, 2 * (k + u) + ((lane >> 3) & 1)), kf[u]);
#pragma unroll
                    for (int u = 0; u < F::kDeep; ++u) {
                        mma<T>(sums[u % kSums][t], qf[k + u], kf[u][0], kf[u][1]);
                        mma<T>(sums[u % kSums][t + 1], qf[k + u], kf[u][2], kf[u][3]);
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < kEights; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[t][e] = (kSums == 2 ? sums[0][t][e] + sums[kSums - 1][t][e] : sums[0][t][e]) * a.scale2;
            if (there != (unsigned)((1ull << kSub) - 1) || k0 < all_lo || k0 + kSub > all_hi) {
#pragma unroll
                for (int t = 0; t < kEights; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int at = 8 * t + 2 * quad + (e & 1), key = k0 + at, h = e >> 1;
                        if (!(key >= lo[h] && key < hi[h] && (there >> at & 1))) s[t][e] = -INFINITY;
                    }
            }
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int t = 0; t < kEights; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) mx[e >> 1] = fmaxf(mx[e >> 1], s[t][e]);
            if (a.scores) {
                float *sc =
                    a.scores + (((int64_t)b * kv.heads + hk) * a.max_tiles * kTile + k0 - sh.first) * a.score_rows + r0;
#pragma unroll
                for (int t = 0; t < kEights; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = 8 * t + 2 * quad + (e & 1), r = grp + 8 * (e >> 1);
                        if (r < rows) sc[key * a.score_rows + r] = s[t][e];
                    }
            }
            // the maximum is raised where a score exceeds it by more than kHeadroom (in steps of
            // exp2): a P of 2^8 and its sum have the same relative rounding
            if (__any_sync(kFull, mx[0] - m[0] > kHeadroom || mx[1] - m[1] > kHeadroom)) {  // -inf - -inf: not
                float w[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    mx[h] = fmaxf(mx[h], __shfl_xor_sync(kFull, mx[h], 1));
                    mx[h] = fmaxf(mx[h], __shfl_xor_sync(kFull, mx[h], 2));
                    mx[h] = fmaxf(m[h], mx[h]);
                    w[h] = exp2_fast(m[h] - (mx[h] == -INFINITY ? 0.0f : mx[h]));
                    l[h] *= w[h];
                    m[h] = mx[h];
                }
#pragma unroll
                for (int d = 0; d < DP / 8; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d][e] *= w[e >> 1];
            }
            const float shift[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
#pragma unroll
            for (int t = 0; t < kEights; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[t][e] = exp2_fast(s[t][e] - shift[e >> 1]);
                    l[e >> 1] += s[t][e];
                }
#pragma unroll
            for (int g = 0; g < kSub / 16; ++g) {
                uint32_t ph[4], pl[4];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    split<T>(s[2 * g + t][0], s[2 * g + t][1], ph[2 * t], pl[2 * t]);
                    split<T>(s[2 * g + t][2], s[2 * g + t][3], ph[2 * t + 1], pl[2 * t + 1]);
                }
#pragma unroll
                for (int d = 0; d < DP / 16; d += 2) {
                    uint32_t vf[2][4];
                    const int r = 16 * g + (lane & 15);
#pragma unroll
                    for (int u = 0; u < 2; ++u) ldsm4_t(st + F::kHalf + F::at(r, 2 * (d + u) + (lane >> 4)), vf[u]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) mma<T>(o[2 * d + u], ph, vf[u / 2][2 * (u & 1)], vf[u / 2][2 * (u & 1) + 1]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) mma<T>(o[2 * d + u], pl, vf[u / 2][2 * (u & 1)], vf[u / 2][2 * (u & 1) + 1]);
                }
            }
        }
        copy_wait<0>();
        // ---- join the warps through shared memory (the ring is empty)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(kFull, l[h], 1);
            l[h] += __shfl_xor_sync(kFull, l[h], 2);
            if (quad == 0) s_stat[warp][grp + 8 * h] = make_float2(m[h], l[h]);
        }
        __syncthreads();
        float *all = reinterpret_cast<float *>(smem);
        constexpr int kPitch = DP + 8;
#pragma unroll
        for (int d = 0; d < DP / 8; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2 *>(all + (warp * kRows + grp + 8 * h) * kPitch + 8 * d + 2 * quad) =
                    make_float2(o[d][2 * h], o[d][2 * h + 1]);
        __syncthreads();
        const bool whole = nt == sh.tiles;
        const int slot = 2 * (int)blockIdx.x + (t0 == 0 ? 1 : 0);
        for (int id = tid; id < rows * (DP / 4); id += F::kThreads) {
            const int r = id / (DP / 4), d = 4 * (id % (DP / 4));
            float M = -INFINITY, L = 0.0f;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < W; ++w) M = fmaxf(M, s_stat[w][r].x);
            const float ref = M == -INFINITY ? 0.0f : M;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float2 z = s_stat[w][r];
                const float e = exp2_fast(z.x - ref);
                const float4 x = *reinterpret_cast<const float4 *>(all + (w * kRows + r) * kPitch + d);
                L += z.y * e;
                v.x += x.x * e;
                v.y += x.y * e;
                v.z += x.z * e;
                v.w += x.w * e;
            }
            if (!whole) {
                *reinterpret_cast<float4 *>(a.part + ((int64_t)slot * kRows + r) * DP + d) = v;
                if (d == 0) a.stat[(int64_t)slot * kRows + r] = make_float2(M, L);
                continue;
            }
            const float inv = inverse(M, L);
            put_row<T>(a, row0, hk, r0 + r, d, v, inv);
            const int t = row0 + (r0 + r) / a.G, h = hk * a.G + (r0 + r) % a.G;
            if (d == 0) {
                if (j.lse) j.lse[(int64_t)t * j.Hq + h] = kLn2 * (M + log2f(L));
                if (a.norm) a.norm[(int64_t)t * j.Hq + h] = make_float2(M, inv);
            }
        }
        __syncthreads();
    }
}

// What is left once every part is there.  The first CTA of a (sequence, key head) puts
// the parts of several CTAs together, in the order of the keys; the others add to the
// mass of kMassKeys keys each, a thread a key: sum over the rows of exp2(score -
// maximum) / sum.
// (Joining alone takes more threads: of 38 parts a key head 89.8 us a call with 512
// where 93.5 with 256; the mass wants more CTAs.)
constexpr int kMassKeys = 1024;
template <typename T, int DP, int kFinThreads>
__device__ __forceinline__ void few_finish(const FewArgs &a) {
    __shared__ float2 s_norm[kFewRowsWhole];
    extern __shared__ __align__(16) float s_weight[];  // [rows][parts], then the groups' sums
    const AttendJob &j = a.j;
    const KvView &kv = a.kv;
    // (one long dimension: the others end at 65535)
    const int nth = (int)(blockIdx.x % a.finishers), item = (int)(blockIdx.x / a.finishers);
    const int b = blockIdx.z, hk = item % kv.heads, rt = item / kv.heads, tid = threadIdx.x;
    const Share sh = share(a, b);
    const int first = sh.first + (nth - 1) * kMassKeys, len = sh.len;  // of the keys
    const bool idle = !sh.work || (nth > 0 ? rt > 0 || first >= len : rt >= sh.rts || a.whole);
    if (idle) return;
    const int64_t total = a.before[kv.B], C = min((int64_t)a.C, total);
    const int row0 = sh.row0;
    // the CTAs that had parts of row tile t
    auto owners = [&](int t, int &c0, int &c1) {
        const int64_t i0 = a.before[b] + ((int64_t)hk * sh.rts + t) * sh.units, i1 = i0 + sh.units;
        c0 = owner(a.whole ? i0 : i0 + kSetUp, total, C);
        c1 = a.whole ? c0 : owner(i1 - 1, total, C);
    };
    if (nth == 0) {
        int c0, c1;
        owners(rt, c0, c1);
        if (c0 == c1) return;
        const int r0 = rt * kRows, rows = min(kRows, sh.rows - r0);
        auto slot = [&](int c) { return (int64_t)(2 * c + (c == c0 ? 1 : 0)) * kRows; };
        // the parts' weights, a warp a row; then their sum, with threads enough for
        // several parts at a time
        const int ns = c1 - c0 + 1, lane = tid & 31;
        for (int r = tid >> 5; r < rows; r += kFinThreads / 32) {
            float M = -INFINITY, L = 0.0f;
            for (int i = lane; i < ns; i += 32) M = fmaxf(M, a.stat[slot(c0 + i) + r].x);
#pragma unroll
            for (int o = 16; o; o >>= 1) M = fmaxf(M, __shfl_xor_sync(kFull, M, o));
            const float ref = M == -INFINITY ? 0.0f : M;
            for (int i = lane; i < ns; i += 32) {
                const float2 z = a.stat[slot(c0 + i) + r];
                const float e = exp2_fast(z.x - ref);
                L += z.y * e;
                s_weight[r * ns + i] = e;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) L += __shfl_xor_sync(kFull, L, o);
            if (lane == 0) {
                s_norm[r] = make_float2(M, inverse(M, L));
                if (j.lse)
                    j.lse[(int64_t)(row0 + (r0 + r) / a.G) * j.Hq + hk * a.G + (r0 + r) % a.G] = kLn2 * (M + log2f(L));
            }
        }
        __syncthreads();
        const int cols = rows * (DP / 4), groups = max(1, kFinThreads / cols);
        float4 *s_sum = reinterpret_cast<float4 *>(s_weight + (rows * ns + 3) / 4 * 4);
        for (int id = tid; id < cols * groups; id += kFinThreads) {
            const int g = id / cols, col = id - g * cols, r = col / (DP / 4), d = 4 * (col % (DP / 4));
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
            for (int i = g; i < ns; i += groups) {
                const float e = s_weight[r * ns + i];
                const float4 x = *reinterpret_cast<const float4 *>(a.part + (slot(c0 + i) + r) * DP + d);
                v.x += x.x * e;
                v.y += x.y * e;
                v.z += x.z * e;
                v.w += x.w * e;
            }
            if (groups > 1) {
                s_sum[id] = v;
                continue;
            }
            put_row<T>(a, row0, hk, r0 + r, d, v, s_norm[r].y);
        }
        if (groups == 1) return;
        __syncthreads();
        if (tid < cols) {
            float4 v = s_sum[tid];
            for (int g = 1; g < groups; ++g) {
                const float4 x = s_sum[g * cols + tid];
                v.x += x.x;
                v.y += x.y;
                v.z += x.z;
                v.w += x.w;
            }
            const int r = tid / (DP / 4);
            put_row<T>(a, row0, hk, r0 + r, 4 * (tid % (DP / 4)), v, s_norm[r].y);
        }
        return;
    }
    if (tid < kFewRowsWhole) {
        float2 z = make_float2(0.0f, 0.0f);  // rows that are not there, or see nothing, add nothing
        if (tid < sh.rows) {
            int c0, c1;
            owners(tid / kRows, c0, c1);
            if (c0 == c1) {
                z = a.norm[(int64_t)(row0 + tid / a.G) * j.Hq + hk * a.G + tid % a.G];
            } else {
                auto at = [&](int c) { return (int64_t)(2 * c + (c == c0 ? 1 : 0)) * kRows + tid % kRows; };
                float M = -INFINITY, L = 0.0f;
                for (int c = c0; c <= c1; ++c) M = fmaxf(M, a.stat[at(c)].x);
                for (int c = c0; c <= c1; ++c) {
                    const float2 p = a.stat[at(c)];
                    L += p.y * exp2_fast(p.x - (M == -INFINITY ? 0.0f : M));
                }
                z = make_float2(M, inverse(M, L));
            }
            if (z.x == -INFINITY) z = make_float2(0.0f, 0.0f);
        }
        s_norm[tid] = z;
    }
    __syncthreads();
    const float *scores = a.scores + ((int64_t)b * kv.heads + hk) * (a.max_tiles << a.tile_log) * a.score_rows;
#pragma unroll
    for (int k = 0; k < kMassKeys; k += kFinThreads) {
        const int key = first + k + tid;
        int page, at;
        if (key >= len || !kv.place(b, key, page, at)) continue;
        float sum = 0.0f;
        for (int r = 0; r < sh.rows; r += 4) {
            const float4 s = *reinterpret_cast<const float4 *>(scores + (int64_t)(key - sh.first) * a.score_rows + r);
            const float2 z0 = s_norm[r], z1 = s_norm[r + 1], z2 = s_norm[r + 2], z3 = s_norm[r + 3];
            sum += exp2_fast(s.x - z0.x) * z0.y;
            if (r + 1 < sh.rows) sum += exp2_fast(s.y - z1.x) * z1.y;
            if (r + 2 < sh.rows) sum += exp2_fast(s.z - z2.x) * z2.y;
            if (r + 3 < sh.rows) sum += exp2_fast(s.w - z3.x) * z3.y;
        }
        *kv.mass_at(page, at, hk) += sum;
    }
}
template <typename T, int DP, int kFinThreads>
__global__ void __launch_bounds__(kFinThreads) k_few_finish(const __grid_constant__ FewArgs a) {
    follow(a.j.beside);
    few_finish<T, DP, kFinThreads>(a);
    end_after(a.j.beside);
}


// Whether a CTA takes all keys of a row tile, which saves the finishing kernel: of up to
// 512 keys, or 1024 of narrow heads, whose steps are of 32 (8 heads of 64 and of 128 over
// 1000 keys, 8 sequences: 8.0 and 12.3 us a call, in parts 10.2 and 12.9; 64 sequences
// 22 and 41, in parts 22 and 34).
bool few_whole(const KvView &kv) {
    return (int64_t)kv.max_pages * kv.ps.d <= (kv.dim <= 96 ? 2 * kFewWholeKeys : kFewWholeKeys);
}

template <typename T, int DP>
cudaError_t few(const AttendJob &j, const KvView &kv, cudaStream_t s, bool finish) {
    if (finish && !j.accumulate && few_whole(kv)) return cudaSuccess;  // nothing is in parts
    FewArgs a{};
    a.j = j;
    a.kv = kv;
    a.G = j.Hq / kv.heads;
    a.whole = few_whole(kv);
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int row_tiles = (int)((std::min<int64_t>(j.few_rows, (int64_t)j.max_new * a.G) + kRows - 1) / kRows);
    const bool wide = a.whole && (int64_t)kv.B * kv.heads * row_tiles <= sms;
    a.C = wide ? sms : 2 * sms;
    a.scale2 = j.scale * kLog2e;
    const int tile = wide ? Few<DP, 8>::kTile : Few<DP, 4>::kTile;
    while (1 << a.tile_log < tile) ++a.tile_log;
    const int64_t seen = seen_keys(j, kv, tile);
    a.max_tiles = (int)((seen + tile - 1) / tile);
    a.score_rows = score_rows(j, kv);
    auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
    const size_t parts = up((size_t)2 * a.C * kRows * DP * sizeof(float)), stats = up((size_t)2 * a.C * kRows * sizeof(float2));
    const size_t befores = up((size_t)(kv.B + 1) * sizeof(int64_t));
    const size_t norms = j.accumulate ? up((size_t)kv.T * j.Hq * sizeof(float2)) : 0;
    const size_t scores =
        j.accumulate ? (size_t)kv.B * kv.heads * a.max_tiles * tile * a.score_rows * sizeof(float) : 0;
    void *buf = nullptr;
    cudaError_t e = stream_scratch(kScratchAttention, parts + stats + befores + norms + scores, s, &buf);
    if (e != cudaSuccess) return e;
    char *at = static_cast<char *>(buf);
    a.part = reinterpret_cast<float *>(at);
    a.stat = reinterpret_cast<float2 *>(at + parts);
    a.before = reinterpret_cast<int64_t *>(at + parts + stats);
    if (j.accumulate) {
        a.norm = reinterpret_cast<float2 *>(at + parts + stats + befores);
        a.scores = reinterpret_cast<float *>(at + parts + stats + befores + norms);
    }
    auto launch_rows = [&](auto kern, int threads, int smem) {
        const cudaError_t e =
            func_attr(reinterpret_cast<const void *>(kern), cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        return e != cudaSuccess ? e : launch_dependent(kern, dim3((unsigned)a.C), threads, smem, s, a);
    };
    if (!finish)
        return wide ? launch_rows(k_few<T, DP, 8>, Few<DP, 8>::kThreads, Few<DP, 8>::kSmem)
                    : launch_rows(k_few<T, DP, 4>, Few<DP, 4>::kThreads, Few<DP, 4>::kSmem);
    // (with accumulate fewer than 2^20 in all, as kMostScores bounds them)
    a.finishers = 1 + (j.accumulate ? (unsigned)((seen + kMassKeys - 1) / kMassKeys) : 0u);
    const dim3 grid(a.finishers * (unsigned)(kv.heads * (a.whole ? 1 : row_tiles)), 1, (unsigned)kv.B);
    auto launch = [&](auto kern, int threads) {
        return launch_dependent(kern, grid, threads, (size_t)(kRows * a.C + 4) * sizeof(float) + threads * sizeof(float4), s,
                                a);
    };
    return j.accumulate ? launch(k_few_finish<T, DP, 256>, 256) : launch(k_few_finish<T, DP, 512>, 512);
}

// The kernel of the rows, or the one that finishes them.
cudaError_t few_by_type(const AttendJob &j, const KvView &kv, cudaStream_t s, bool finish) {
    const bool bf = j.type == PVMVMD_BF16;
    if (kv.dim <= 64) return bf ? few<__nv_bfloat16, 64>(j, kv, s, finish) : few<__half, 64>(j, kv, s, finish);
    if (kv.dim <= 96) return bf ? few<__nv_bfloat16, 96>(j, kv, s, finish) : few<__half, 96>(j, kv, s, finish);
    return bf ? few<__nv_bfloat16, 128>(j, kv, s, finish) : few<__half, 128>(j, kv, s, finish);
}

}  // namespace

cudaError_t launch_attention_few(const AttendJob &j, const KvView &kv, cudaStream_t s) {
    return few_by_type(j, kv, s, false);
}
cudaError_t launch_attention_few_finish(const AttendJob &j, const KvView &kv, cudaStream_t s) {
    return few_by_type(j, kv, s, true);
}

}  // namespace pv
