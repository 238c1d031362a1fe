// Attention of many new rows (tokens of a chunk x query heads of a key head) over a
// paged cache, on the tensor cores: 8192 tokens of 32 heads of 128 over 24576 keys in
// 1.71-1.74 ms, 1.6 PFLOP/s, which the power cap bounds; where there are few items, what
// a CTA does before and after its tiles (5 us).
//
// A CTA takes 256 rows of one sequence and key head, token by token with the heads
// of a token side by side, as two tiles of 128, and walks the keys that they see in
// tiles of 128:
//     S = Q K^T  (128 x 128, fp32 in TMEM),  P = exp2(scale2 (S - m)),  O += P V.
// P goes back to TMEM as 16-bit values in the place of its S, from where the second
// product reads it as its A operand; O (128 x D) stays in TMEM.
//
// Warps (384 threads):
//   0-3, 4-7  the softmax of tile 0, of tile 1: a thread holds one row of S.  While
//             one tile's is under way the tensor cores work for the other.
//   8         issues the MMAs
//   9-11      copy Q, then tiles of K and V through a ring, gathering the rows of
//             their pages.  Each takes whole tiles: the fence that shows a tile to
//             the MMAs waits for all that its warp has in flight (a third of every
//             tile each, three tiles ahead, took 3.6 us for 256 rows and 128 keys)
// The running maximum m is raised only where S exceeds it by more than 2^8 (in
// steps of exp2), so that O is rescaled seldom, by the softmax warps themselves:
// P stays below 2^8, and its sum and O are exact multiples of what they would be.
// P is rounded to the cache's 16-bit type (2^-9 of each at most, for bf16), as the
// MMA takes both operands in one type; the sum of a row is that of the 32-bit values.
#include <algorithm>
#include <climits>
#include <cmath>

#include "attention.cuh"

namespace pv {
namespace {

constexpr int kCRows = 2 * kCM;      // rows per CTA
constexpr float kCHeadroom = 8.0f;   // log2 of the largest P

struct ChunkArgs {
    AttendJob j;
    KvView kv;
    float4 *part;   // [items][splits][DP / 4][256] normalised partial outputs
    float *stat;    // [items][splits][256] log2 of their sums
    float scale2;   // |scale| log2(e)
    int G, splits, negative;
    int box;        // keys per TMA box, 0: the pages are not such that boxes fit them
    bool q_box;     // a tile of rows is a TMA box (see rows_map)
};

template <int DP>
struct Chunk {
    static constexpr int kSlabs = DP / 64;             // 128-byte wide parts of a tile's rows
    static constexpr int kSlab = kCN * 128;            // bytes
    static constexpr int kTileBytes = kSlabs * kSlab;  // of Q, K and V alike
    static constexpr int kStages = DP == 128 ? 5 : 8;
    static constexpr int kSmem = (2 + kStages) * kTileBytes + 1024;
    static constexpr int kO = 2 * kCN;                 // TMEM column of O
};

// V as the B operand: D (the N dimension) is contiguous.  64 values of D are a
// swizzled 128-byte row, 8 keys 1024 bytes (stride offset), the next 64 values a
// slab further (leading offset).
__device__ __forceinline__ uint64_t sw128_desc_mn(uint32_t saddr, uint32_t slab) {
    return (sw128_desc(saddr) & ~((uint64_t)0x3FFFu << 16)) | (uint64_t)(slab >> 4) << 16;
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
// A row's log2 of its sum.  The scratch copy is negative, to be added to scores, and
// -infinity also for a row that sees nothing.
__device__ __forceinline__ void row_sum(const AttendJob &j, int64_t row, float lse2) {
    if (j.lse) j.lse[row] = kLn2 * lse2;
    if (j.lse2) j.lse2[row] = lse2 == -INFINITY ? lse2 : -lse2;
}

// ---------------------------------------------------------------- work
__device__ __forceinline__ int chunk_tiles(const ChunkArgs &a, int b) {
    const int rows = many_rows(a.kv, a.j.few_rows, a.G, b);
    return (rows + kCRows - 1) / kCRows;
}
// Item `idx` (row tile and key head of a sequence; the last tiles, which see most
// keys, come first) and its share of the keys.
struct ChunkItem {
    int b, hk, row0, rows;       // rows of the sequence and key head, of this item
    int len, n, t0;              // cached and new tokens, the first of these
    int kt0, kt1;                // key tiles of the item
    int per, parts;              // key tiles of a split, splits that have any
    int64_t slot;                // of the item, for partial results
};
__device__ __forceinline__ bool chunk_item(const ChunkArgs &a, int idx, ChunkItem &it) {
    const KvView &kv = a.kv;
    // lengths, which are wanted once the sequence is found
    asm volatile("prefetch.global.L1 [%0];" ::"l"(kv.lens + min((int)threadIdx.x, kv.B - 1)));
    const int hk = idx % kv.heads;
    const int64_t rank = idx / kv.heads;
    const Found f = find<kCThreads>(kv.B, [&](int b) { return (int64_t)chunk_tiles(a, b); },
                                    [&](int64_t total) { return total - 1 - rank; });
    if (f.b < 0) return false;
    it.b = f.b;
    it.hk = hk;
    it.len = kv.len(f.b);
    it.n = kv.news(f.b);
    it.t0 = kv.first(f.b);
    it.row0 = (int)(f.total - 1 - rank - f.before) * kCRows;
    it.rows = min(kCRows, it.n * a.G - it.row0);
    const int at0 = it.len - it.n + it.row0 / a.G, at1 = it.len - it.n + (it.row0 + it.rows - 1) / a.G;
    const int hi = a.j.causal ? max(0, min(it.len, at1 + 1)) : it.len;
    const int lo = a.j.window > 0 && at0 >= a.j.window ? at0 - a.j.window + 1 : 0;
    it.kt0 = min(lo, hi) / kCN;
    it.kt1 = max(it.kt0 + 1, (hi + kCN - 1) / kCN);  // a tile at least, if all of it is hidden
    const int n = it.kt1 - it.kt0;
    it.per = (n + a.splits - 1) / a.splits;
    it.parts = (n + it.per - 1) / it.per;
    it.slot = (int64_t)idx * a.splits;
    return true;
}

// ---------------------------------------------------------------- main kernel
template <typename T, int DP>
__device__ __forceinline__ void chunk_split(const ChunkArgs &a, const CUtensorMap &q_map, const CUtensorMap &k_map,
                                            const CUtensorMap &v_map, uint32_t *err) {
    using C = Chunk<DP>;
    constexpr int kSt = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t q_full, kv_full[kSt], kv_empty[kSt], s_full[2], p_full[2][2], o_done[2], mma_done;
    __shared__ uint32_t s_tmem;
    // Whether keys of tile i are not there, at i % kGaps.  K's tiles lie two places apart in
    // the ring, and the place of tile i is free once the MMAs on it are through, which the
    // softmax warps' reading of its flag is not.  Tile i + 8 waits for the place of tile
    // i + 4 or a later one, whose MMAs follow P of tile i + 3, and with it that reading.
    constexpr int kGaps = 8;
    static_assert(kSt <= kGaps, "a place is taken again by tile i + kGaps / 2 at the earliest");
    __shared__ bool s_gap[kGaps];
    const AttendJob &j = a.j;
    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(kFull, tid >> 5, 0);
    ChunkItem it;
    if (!chunk_item(a, blockIdx.x, it)) return;
    const int split = blockIdx.y;
    if (split >= it.parts) return;
    const int kt0 = it.kt0 + split * it.per, nk = min(it.kt1, kt0 + it.per) - kt0;
    const int used = it.rows > kCM ? 2 : 1;  // tiles with rows

    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t qbase = base, ring = base + 2 * C::kTileBytes;
    if (tid == 0) {
        mbar_init(&q_full, a.q_box ? 1 : 8);
        mbar_init(&mma_done, 1);
        for (int s = 0; s < kSt; ++s) {
            mbar_init(&kv_full[s], 1);
            mbar_init(&kv_empty[s], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&s_full[t], 1);
            mbar_init(&p_full[t][0], 4);
            mbar_init(&p_full[t][1], 4);
            mbar_init(&o_done[t], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    // ring places of the tiles: K0, K1, V0, K2, V1, ..., the last V
    const int places = 2 * nk;
    auto place_k = [&](int i) { return i == 0 ? 0 : 2 * i - 1; };
    auto place_v = [&](int i) { return min(2 * i + 2, places - 1); };

    if (warp < 8) {
        // ------------------------------------------------ softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kCSoftRegs));
        const int tile = warp >> 2, r = tile * kCM + (warp & 3) * 32 + lane;
        const bool real = r < it.rows;
        const int at = it.len - it.n + (it.row0 + r) / a.G;
        const int hi = !real ? INT_MAX : j.causal ? min(it.len, at + 1) : it.len;
        const int lo = real && j.window > 0 && at >= j.window ? at - j.window + 1 : 0;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        if (!a.q_box) {  // the warp's rows of Q
            const TileCopy<DP> q(lane, kv.dim);
            q.template copy<1>(qbase + tile * C::kTileBytes, static_cast<const char *>(j.q), [&](int, int64_t &off) {
                off = (int64_t)(it.t0 + (it.row0 + r) / a.G) * j.q_token +
                      (int64_t)(it.hk * a.G + (it.row0 + r) % a.G) * j.q_head;
                return real;
            }, (warp & 3) * 32);
            q.arrive(&q_full);
        }
        const uint32_t ts = tmem + lanes + (uint32_t)(tile * kCN), to = tmem + lanes + (uint32_t)(C::kO + tile * DP);
        float m = -INFINITY, l = 0.0f;
        bool ok = true;
        for (int i = 0; i < nk && tile < used; ++i) {
            if (!mbar_wait_warp(&s_full[tile], i & 1, err, kWaitNs)) {
                ok = false;
                break;
            }
            tc_fence_after();
            float s[kCN];
#pragma unroll
            for (int c = 0; c < kCN / 32; ++c) tmem_ld32_async(ts + 32 * c, s + 32 * c);
            const int k0 = (kt0 + i) * kCN;
            const bool gap = s_gap[i % kGaps];
            tmem_ld_wait();
            if (__any_sync(kFull, k0 < lo || hi - kCN < k0) || gap) {
#pragma unroll
                for (int c = 0; c < kCN / 32; ++c) {
                    // bits of the keys that this row sees
                    const int from = lo - k0 - 32 * c, to = hi - k0 - 32 * c;
                    uint32_t see = to >= 32 ? kFull : to <= 0 ? 0u : (1u << to) - 1u;
                    if (from > 0) see = from >= 32 ? 0u : see & ~((1u << from) - 1u);
                    if (gap) {
                        const int key = k0 + 32 * c + lane;
                        int page, slot;
                        see &= __ballot_sync(kFull, key < it.len && kv.place(it.b, key, page, slot));
                    }
                    if (__any_sync(kFull, see != kFull)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[32 * c + e] = see >> e & 1 ? s[32 * c + e] : -INFINITY;
                    }
                }
            }
            float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
            for (int e = 4; e < kCN; e += 8)
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = e + 2 * k + 1 < kCN ? max3(mx[k], s[e + 2 * k], s[e + 2 * k + 1]) : mx[k];
            const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
            // (-inf - -inf: not; rows that are not of the sequence have no say, as they see anything)
            if (__any_sync(kFull, real && (top - m) * a.scale2 > kCHeadroom)) {
                const float mn = fmaxf(m, top), w = m == -INFINITY ? 0.0f : exp2_fast((m - mn) * a.scale2);
                m = mn;
                l *= w;
                if (i > 0) {
                    if (!mbar_wait_warp(&o_done[tile], (i - 1) & 1, err, kWaitNs)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < DP / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(to + 32 * c, o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * w);
                        tmem_st32(to + 32 * c, o);
                    }
                }
            }
            const float shift = m == -INFINITY ? 0.0f : -m * a.scale2;
            const uint64_t scale_2 = pair(a.scale2, a.scale2), shift_2 = pair(shift, shift);
            uint64_t sum[2] = {0u, 0u};
            // P in two halves, so that the MMAs on the first run while the second is formed
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    float x, y;
                    unpair(fma2(pair(s[64 * c + 2 * e], s[64 * c + 2 * e + 1]), scale_2, shift_2), x, y);
                    x = exp2_fast(x);
                    y = exp2_fast(y);
                    sum[e & 1] = add2(sum[e & 1], pair(x, y));
                    p[e] = pack(x, y, T{});
                }
                tmem_st32(ts + 32 * c, p);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[tile][c]);
            }
            float x, y;
            unpair(add2(sum[0], sum[1]), x, y);
            l += x + y;
        }
        // ------------------------------------------------ output
        if (ok && tile < used && mbar_wait_warp(&o_done[tile], (nk - 1) & 1, err, kWaitNs)) {
            tc_fence_after();
            const int t = it.t0 + (it.row0 + r) / a.G, h = it.hk * a.G + (it.row0 + r) % a.G;
            const float inv = inverse(m, l), lse2 = m == -INFINITY ? (l != l ? l : m) : m * a.scale2 + log2f(l);
            const int64_t part = it.slot + split;
            // Rows go through the memory of the warp's rows of Q, which no MMA reads any more, so
            // that a row's 16-byte pieces leave from neighbouring lanes (a lane a row, 2048
            // tokens over 8192 keys: 164 us a call, so 160).
            constexpr int kPieces = DP / 8;
            const uint32_t rows = qbase + tile * C::kTileBytes + (warp & 3) * 32 * 2 * DP;
            auto piece = [&](int row, int p) { return rows + (uint32_t)(row * kPieces + (p ^ (row & 7))) * 16; };
#pragma unroll 1
            for (int c = 0; c < DP / 32; ++c) {
                float o[32];
                tmem_ld32_async(to + 32 * c, o);
                tmem_ld_wait();
                if (it.parts > 1) {
                    if (!real) continue;
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        a.part[(part * (DP / 4) + 8 * c + e / 4) * kCRows + r] =
                            make_float4(o[e] * inv, o[e + 1] * inv, o[e + 2] * inv, o[e + 3] * inv);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        shared_store16(piece(lane, 4 * c + e / 8), pack(o[e] * inv, o[e + 1] * inv, T{}),
                                       pack(o[e + 2] * inv, o[e + 3] * inv, T{}), pack(o[e + 4] * inv, o[e + 5] * inv, T{}),
                                       pack(o[e + 6] * inv, o[e + 7] * inv, T{}));
                }
            }
            if (it.parts == 1) {
                __syncwarp();
                const int64_t orow = t * j.o_token + h * j.o_head;
                const int ch = lane % kPieces;
                char *out = static_cast<char *>(j.out) + 16 * ch;
#pragma unroll 4
                for (int u = 0; u < kPieces; ++u) {
                    const int row = u * (32 / kPieces) + lane / kPieces;
                    const int64_t at = __shfl_sync(kFull, orow, row);
                    if (r - lane + row < it.rows && 8 * ch < kv.dim)
                        *reinterpret_cast<uint4 *>(out + at) = shared_load16(piece(row, ch));
                }
            }
            if (real) {
                if (it.parts > 1)
                    a.stat[part * kCRows + r] = lse2;
                else
                    row_sum(j, (int64_t)t * j.Hq + h, lse2);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCOtherRegs));
        if (warp == 8) {
            // ------------------------------------------------ MMA issuer
            const uint32_t id_s = chunk_idesc<T>(kCN) | (a.negative ? 1u << 13 : 0u), id_o = chunk_idesc<T>(DP) | 1u << 16;
            auto stage = [&](int place) { return ring + (uint32_t)(place % kSt) * C::kTileBytes; };
            auto full = [&](int place) { return mbar_wait_warp(&kv_full[place % kSt], (place / kSt) & 1, err, kWaitNs); };
            auto scores = [&](int t, int i) {  // S = Q K^T
                const uint64_t ad = sw128_desc(qbase + t * C::kTileBytes), bd = sw128_desc(stage(place_k(i)));
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k) {
                        const uint32_t off = (uint32_t)((k >> 2) * (C::kSlab >> 4) + (k & 3) * 2);
                        mma_ss(tmem + t * kCN, ad + off, bd + off, id_s, k > 0);
                    }
                    commit(&s_full[t]);
                }
                __syncwarp();
            };
            auto output = [&](int t, int i, int half) {  // O += P V, 64 keys
                const uint64_t bd = sw128_desc_mn(stage(place_v(i)), C::kSlab);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kCN / 32; ++k) {
                        const int kk = half * (kCN / 32) + k;
                        mma_ts(tmem + C::kO + t * DP, tmem + t * kCN + 8 * kk, bd + (uint32_t)(kk * (2048 >> 4)), id_o,
                               i > 0 || kk > 0);
                    }
                    if (half) commit(&o_done[t]);
                }
                __syncwarp();
            };
            auto release = [&](int place) {
                if (elect_one()) commit(&kv_empty[place % kSt]);
                __syncwarp();
            };
            bool ok = mbar_wait_warp(&q_full, 0, err, kWaitNs) && full(0);
            if (ok) {
                tc_fence_after();
                for (int t = 0; t < used; ++t) scores(t, 0);
                release(0);
            }
            for (int i = 0; i < nk && ok; ++i) {
                const bool more = i + 1 < nk;
                for (int t = 0; t < used && ok; ++t) {
                    ok = t || full(place_v(i));
                    for (int half = 0; half < 2 && ok; ++half) {
                        ok = mbar_wait_warp(&p_full[t][half], i & 1, err, kWaitNs);
                        if (!ok) break;
                        tc_fence_after();
                        output(t, i, half);
                    }
                    if (!ok) break;
                    if (!more) continue;
                    ok = t || full(place_k(i + 1));
                    if (!ok) break;
                    tc_fence_after();
                    scores(t, i + 1);
                }
                if (!ok) break;
                if (more) release(place_k(i + 1));
                release(place_v(i));
            }
            // every MMA is through before the memory that it reads goes
            if (elect_one()) commit(&mma_done);
            __syncwarp();
            mbar_wait_warp(&mma_done, 0, err, kWaitNs);
        } else {
            // ------------------------------------------------ copies
            const int w = warp - 9;
            const TileCopy<DP> tile(lane, kv.dim);
            if (a.q_box && w == 0) {
                if (lane == 0) {
                    mbar_arrive_tx(&q_full, (uint32_t)(used * C::kTileBytes));
                    for (int t = 0; t < used; ++t)
#pragma unroll
                        for (int s = 0; s < C::kSlabs; ++s)
                            tma_load_3d(qbase + t * C::kTileBytes + s * C::kSlab, &q_map, 64 * s, it.hk * a.G,
                                        it.t0 + (it.row0 + t * kCM) / a.G, &q_full);
                }
                __syncwarp();
            }
            // tiles of K and V in turn
            int x = w;
            for (; x < places; x += kCLoaders) {
                const bool values = (x > 0 && x % 2 == 0) || x == places - 1;
                const int i = !values ? (x + 1) / 2 : x == places - 1 ? nk - 1 : x / 2 - 1;
                if (x >= kSt && !mbar_wait_warp(&kv_empty[x % kSt], ((x / kSt) & 1) ^ 1, err, kWaitNs)) break;
                const int64_t ps = values ? kv.v_page : kv.k_page, ss = values ? kv.v_slot : kv.k_slot,
                              hs = it.hk * (values ? kv.v_head : kv.k_head);
                const int key0 = (kt0 + i) * kCN;
                // (what is behind the end must be zero where a P of 0 meets it)
                if (a.box && (!values || key0 + kCN <= it.len)) {
                    // (before the barrier that the copy itself completes)
                    if (!values && lane == 0) s_gap[i % kGaps] = false;
                    __syncwarp();
                    if (tile.fetch(ring + (uint32_t)(x % kSt) * C::kTileBytes, values ? &v_map : &k_map, a.box, kv, it.b,
                                   it.hk, key0, it.len, &kv_full[x % kSt]))
                        continue;
                }
                bool gap = false;
                tile.copy(ring + (uint32_t)(x % kSt) * C::kTileBytes, values ? kv.V : kv.K, [&](int rr, int64_t &off) {
                    const bool is = key_place(kv, it.b, it.len, key0 + rr, ps, ss, off);
                    gap |= key0 + rr < it.len && !is;
                    off += hs;
                    return is;
                });
                gap = __any_sync(kFull, gap);
                if (!values && lane == 0) s_gap[i % kGaps] = gap;
                tile.arrive(&kv_full[x % kSt]);
            }
            // copies in flight complete before the CTA may exit (a tile whose place has
            // been filled again was read, and its barrier is a phase ahead)
            for (int y = x - kCLoaders; y >= 0 && y + kSt >= min(places, x); y -= kCLoaders)
                mbar_wait_warp(&kv_full[y % kSt], (y / kSt) & 1, err, kWaitNs);
            if (w == 0) mbar_wait_warp(&q_full, 0, err, kWaitNs);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}
template <typename T, int DP>
__global__ void __launch_bounds__(kCThreads, 1)
    k_chunk(const __grid_constant__ ChunkArgs a, const __grid_constant__ CUtensorMap q_map,
            const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
            uint32_t *__restrict__ err) {
    follow(a.j.beside);
    chunk_split<T, DP>(a, q_map, k_map, v_map, err);
    end_after(a.j.beside);
}

// Items of several splits: their parts, in the order of the keys.  kJoinRows rows a CTA
// (8 of many parts, else 32; 19 parts of eight items: 58 us a call, with 32 rows 76; 3
// parts of eighty 148 and 141); a thread 4 values of a row, eight rows of four such side
// by side.
template <typename T, int DP, int kJoinRows>
__global__ void __launch_bounds__(kCThreads) k_chunk_join(const __grid_constant__ ChunkArgs a) {
    follow();
    ChunkItem it;
    if (!chunk_item(a, blockIdx.x, it) || it.parts == 1) return;
    const int r0 = blockIdx.y * kJoinRows;
    for (int id = threadIdx.x; id < kJoinRows * (DP / 4); id += kCThreads) {
        const int c4 = (id & 3) | (id / (4 * kJoinRows)) << 2, r = r0 + (id / 4) % kJoinRows;
        if (r >= it.rows) continue;
        float M = -INFINITY, L = 0.0f;
#pragma unroll 4
        for (int p = 0; p < it.parts; ++p) M = fmaxf(M, a.stat[(it.slot + p) * kCRows + r]);
        const float ref = M == -INFINITY ? 0.0f : M;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int p = 0; p < it.parts; ++p) {
            const float e = exp2_fast(a.stat[(it.slot + p) * kCRows + r] - ref);
            const float4 x = a.part[((it.slot + p) * (DP / 4) + c4) * kCRows + r];
            L += e;
            v.x += x.x * e;
            v.y += x.y * e;
            v.z += x.z * e;
            v.w += x.w * e;
        }
        const int t = it.t0 + (it.row0 + r) / a.G, h = it.hk * a.G + (it.row0 + r) % a.G;
        const float inv = inverse(M, L);
        if (4 * c4 < a.kv.dim)
            *reinterpret_cast<uint2 *>(static_cast<char *>(a.j.out) + t * a.j.o_token + h * a.j.o_head + 8 * c4) =
                make_uint2(pack(v.x * inv, v.y * inv, T{}), pack(v.z * inv, v.w * inv, T{}));
        if (c4 == 0) row_sum(a.j, (int64_t)t * a.j.Hq + h, M + log2f(L));
    }
}

template <typename T, int DP>
cudaError_t chunk(const AttendJob &j, const KvView &kv, cudaStream_t s, bool &joined) {
    ChunkArgs a{};
    a.j = j;
    a.kv = kv;
    a.G = j.Hq / kv.heads;
    a.negative = j.scale < 0.0f;
    // (a scale of 0 stays above it, so that hidden scores stay -infinity)
    a.scale2 = std::max(std::fabs(j.scale) * kLog2e, 1e-37f);
    uint32_t *err = library_error_word();
    if (!err) return cudaErrorUnknown;
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    // at most as many row tiles as full ones and one more for each sequence that can have
    // more rows than the kernel of few takes
    const int64_t rows = (int64_t)kv.T * a.G;
    const int64_t tiles = rows / kCRows + std::min<int64_t>(kv.B, rows / (j.few_rows + 1)), items = tiles * kv.heads;
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d, keys = (room + kCN - 1) / kCN;
    // Splits of an item's keys: the number with which all of them would be through first,
    // in turns of one CTA an SM of as many tiles each and as long as kSetUp tiles beside
    // them.  (80 items of up to 120 tiles: 171 us whole, with as many splits as SMs
    // without an item, none; 32 items of 470 tiles want 19.)  No more than kMostParts
    // has room for: the tiles are those of the table, which may be far wider than what is
    // cached, and more items than that have little to gain.
    constexpr int kSetUp = 4, kLeast = 8, kMost = 64;
    a.splits = 1;
    int64_t best = INT64_MAX;
    const int64_t part = (int64_t)kCRows * (DP + 1) * sizeof(float);
    for (int64_t n = 1; n <= kMost && (n == 1 || (n * kLeast <= keys && items * n * part <= kMostParts)); ++n) {
        const int64_t cost = (items * n + sms - 1) / sms * ((keys + n - 1) / n + (n > 1 ? kSetUp + 2 : kSetUp));
        if (cost < best) best = cost, a.splits = (int)n;
    }
    if (items > INT_MAX) return cudaErrorInvalidValue;
    if (a.splits > 1) {
        auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
        const size_t n = (size_t)items * a.splits * kCRows, parts = up(n * DP * sizeof(float));
        void *buf = nullptr;
        const cudaError_t e = stream_scratch(kScratchChunk, parts + n * sizeof(float), s, &buf);
        if (e != cudaSuccess) return e;
        a.part = static_cast<float4 *>(buf);
        a.stat = reinterpret_cast<float *>(static_cast<char *>(buf) + parts);
    }
    CUtensorMap maps[3] = {};
    a.q_box = rows_map(&maps[0], j, kv, a.G);
    a.box = page_box(kv);
    for (int v = 0; a.box && v < 2; ++v)
        if (page_map(&maps[1 + v], kv, v, j.type, a.box) != cudaSuccess) a.box = 0;
    cudaError_t e = func_attr(reinterpret_cast<const void *>(k_chunk<T, DP>), cudaFuncAttributeMaxDynamicSharedMemorySize,
                              Chunk<DP>::kSmem);
    if (e != cudaSuccess) return e;
    e = launch_dependent(k_chunk<T, DP>, dim3((unsigned)items, (unsigned)a.splits), kCThreads, Chunk<DP>::kSmem, s, a,
                         maps[0], maps[1], maps[2], err);
    joined = a.splits > 1;
    if (e == cudaSuccess && joined)
        e = a.splits > 8
                ? launch_dependent(k_chunk_join<T, DP, 8>, dim3((unsigned)items, kCRows / 8), kCThreads, 0, s, a)
                : launch_dependent(k_chunk_join<T, DP, 32>, dim3((unsigned)items, kCRows / 32), kCThreads, 0, s, a);
    return e;
}

}  // namespace

cudaError_t launch_attention_chunk(const AttendJob &j, const KvView &kv, cudaStream_t s, bool &joined) {
    const bool bf = j.type == PVMVMD_BF16;
    if (kv.dim <= 64) return bf ? chunk<__nv_bfloat16, 64>(j, kv, s, joined) : chunk<__half, 64>(j, kv, s, joined);
    return bf ? chunk<__nv_bfloat16, 128>(j, kv, s, joined) : chunk<__half, 128>(j, kv, s, joined);
}

}  // namespace pv
