// The attention weight that keys gather from many new rows: mass_j += sum over the
// rows that see key j of exp2(scale2 q.k_j - lse2), after the attention itself has
// written lse2, each row's log2 of the sum.
//
// Keys are the rows of the product here, so that a thread holds a key, over every second
// tile of rows, and no atomics are needed: S^T = K Q^T.  A CTA keeps two tiles of 128
// keys and walks the rows that see them in tiles of 128 through a ring; each of the
// two has two accumulators in TMEM, so that the tensor cores work on the next tile
// while one is summed.  Few rows over many keys make many short items, so a CTA stays
// and its rows' copies and sums run on from one item to the next (with a barrier at
// each, five chunks of 35 tokens over 13000 keys took 130 us).  Where there are many rows the
// chain of a warp's sums bounds it: 2048 tokens of 32 heads of 128 over 8192 keys 138 us
// beside the attention's 160 (0.87 PFLOP/s, 3.4e12 exp2/s), with the tensor cores, the
// exp2 pipe and the issue slots each busy for about half of that.
#include <algorithm>
#include <climits>
#include <cmath>

#include "attention.cuh"

namespace pv {
namespace {

constexpr int kMKeys = 2 * kCM;  // keys per CTA
constexpr int kShifts = 4;       // ring of the rows' lse2
constexpr int kMostShare = 8;    // CTAs of a cluster
// Warps: 0-15 sum, four of each tile of keys and of the even and of the odd tiles of rows
// (four warps a scheduler, as a warp's sums wait for themselves: with two of them 158
// us); 16 issues the MMAs; 17-19 copy.
constexpr int kMSums = 16, kMThreads = 32 * (kMSums + 4);

struct MassArgs {
    AttendJob j;
    KvView kv;
    float scale2;
    int G, negative;
    FastDiv group, heads;  // G, key heads
    int box;        // keys per TMA box on a page, 0: none (see page_box)
    bool q_box;     // a tile of rows is a TMA box (see rows_map)
};

// ---------------------------------------------------------------- between the CTAs of a cluster
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t peer_addr(const void *p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void peer_store(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void peer_arrive(uint32_t addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// A bounded wait that makes what the peers wrote before their arrivals visible.
__device__ __forceinline__ bool peer_wait(uint64_t *bar, uint32_t parity, uint32_t *err) {
    const uint64_t t0 = global_ns();
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok)
            : "r"(smem_addr(bar)), "r"(parity)
            : "memory");
        if (__all_sync(kFull, ok != 0)) return true;
        if (__any_sync(kFull, global_ns() - t0 > kWaitNs)) break;
    }
    record_error(err, kErrMmaTimeout);
    return false;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int DP>
struct Mass {
    static constexpr int kSlabs = DP / 64, kSlab = kCM * 128, kTileBytes = kSlabs * kSlab;
    static constexpr int kStages = 4;
    static constexpr int kItems = DP == 64 ? 2 : 1;  // whose keys are there at a time
    static constexpr int kSmem = (2 * kItems + kStages) * kTileBytes + 1024;
};

// Keys [first, len) of a sequence that some new row may see, in CTAs' shares.
__device__ __forceinline__ int mass_first(const MassArgs &a, int b) {
    const int at = a.kv.len(b) - a.kv.news(b);
    return a.j.window > 0 && at >= a.j.window ? (at - a.j.window + 1) / kMKeys * kMKeys : 0;
}
__device__ __forceinline__ int mass_shares(const MassArgs &a, int b) {
    return many_rows(a.kv, a.j.few_rows, a.G, b) ? (a.kv.len(b) - mass_first(a, b) + kMKeys - 1) / kMKeys : 0;
}

// Keys [k0, k0 + kMKeys) of a sequence and key head, and this CTA's share of the tiles of
// rows that see any of them: nt from row r0 on, which may be none.
struct MassItem {
    int b, hk, k0, len, old, n, rows, t0, r0, nt;
    // the rows that see a key: [first, last)
    __device__ __forceinline__ int first_row(const MassArgs &a, int key) const {
        return a.j.causal && key > old ? (int)min((int64_t)rows, (int64_t)(key - old) * a.G) : 0;
    }
    __device__ __forceinline__ int last_row(const MassArgs &a, int key) const {
        const int64_t t = a.j.window > 0 ? (int64_t)key + a.j.window - old : n;
        return t >= n ? rows : t <= 0 ? 0 : (int)t * a.G;
    }
};
// A cluster's items in order: one of every `stride` of all (shares of keys and their
// heads), in turns that go forth and back, as later shares have fewer rows.  By whole
// warps.
struct MassWalk {
    int64_t before;  // the shares before sequence b
    int b, mine, stride, rank, size;
    int turn = 0, at = -1;              // sequence that the following are of
    int len = 0, n = 0, t0 = 0, first = 0, shares = 0;
    __device__ __forceinline__ void enter(const MassArgs &a) {
        if (b >= a.kv.B || at == b) return;
        at = b;
        len = a.kv.len(b);
        n = a.kv.news(b);
        t0 = a.kv.first(b);
        first = mass_first(a, b);
        shares = mass_shares(a, b);
    }
    __device__ __forceinline__ bool next(const MassArgs &a, MassItem &it) {
        const KvView &kv = a.kv;
        for (enter(a);;) {
            const int64_t idx = (int64_t)turn * stride + (turn & 1 ? stride - 1 - mine : mine);
            int64_t share;
            if (idx <= INT_MAX) {
                uint32_t q, r;
                a.heads.divmod((uint32_t)idx, q, r);
                share = q;
            } else {
                share = idx / kv.heads;
            }
            // the sequence that holds it, 32 at a time
            while (b < kv.B && share >= before + shares) {
                const int lane = threadIdx.x & 31;
                const int64_t n = b + lane < kv.B ? mass_shares(a, b + lane) : 0;
                int64_t incl = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t v = __shfl_up_sync(kFull, incl, o);
                    if (lane >= o) incl += v;
                }
                const unsigned at = __ballot_sync(kFull, share < before + incl);
                const int to = at ? __ffs(at) - 1 : 32;
                before += at ? __shfl_sync(kFull, incl - n, to) : __shfl_sync(kFull, incl, 31);
                b += to;
                enter(a);
            }
            if (b >= kv.B) return false;
            ++turn;
            it.b = b;
            it.hk = (int)(idx - share * kv.heads);
            it.len = len;
            it.n = n;
            it.t0 = t0;
            it.rows = n * a.G;
            it.old = len - n;
            it.k0 = first + (int)(share - before) * kMKeys;
            it.r0 = it.first_row(a, it.k0) / kCM * kCM;
            const int r1 = it.last_row(a, min(it.k0 + kMKeys, it.len) - 1);
            const int all = r1 > it.r0 ? (r1 - it.r0 + kCM - 1) / kCM : 0;
            if (all == 0) continue;
            const int per = (all + size - 1) / size, from = min(all, rank * per);
            it.r0 += from * kCM;
            it.nt = min(all, from + per) - from;
            return true;
        }
    }
};

template <typename T, int DP>
__global__ void __launch_bounds__(kMThreads, 1)
    k_mass(const __grid_constant__ MassArgs a, const __grid_constant__ CUtensorMap k_map,
           const __grid_constant__ CUtensorMap q_map, uint32_t *__restrict__ err) {
    using C = Mass<DP>;
    constexpr int kSt = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full[kSt], empty[kSt], s_full[2][2], s_empty[2][2], k_full[C::kItems],
        k_empty[C::kItems], mma_done;
    __shared__ __align__(8) uint64_t shift_full[kShifts], shift_empty[kShifts];
    __shared__ __align__(16) float s_shift[kShifts][kCM];
    // the sums of the cluster's other CTAs, in the first one's memory
    __shared__ float s_sums[kMostShare - 1][kMKeys];
    __shared__ __align__(8) uint64_t sums_full, sums_empty;
    // the sums over odd tiles of rows
    __shared__ float s_half[kMKeys];
    __shared__ __align__(8) uint64_t half_full, half_empty;
    __shared__ uint32_t s_tmem;
    const AttendJob &j = a.j;
    const KvView &kv = a.kv;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(kFull, tid >> 5, 0);
    follow(a.j.beside);
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    constexpr int kItems = C::kItems;
    const uint32_t ring = base + 2 * kItems * C::kTileBytes;
    if (tid == 0) {
        for (int s = 0; s < kSt; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int t = 0; t < 4; ++t) {
            mbar_init(&s_full[t >> 1][t & 1], 1);
            mbar_init(&s_empty[t >> 1][t & 1], 4);
        }
        for (int s = 0; s < kItems; ++s) {
            mbar_init(&k_full[s], 2);
            mbar_init(&k_empty[s], 1);
        }
        for (int s = 0; s < kShifts; ++s) {
            mbar_init(&shift_full[s], 32);
            mbar_init(&shift_empty[s], 8);
        }
        mbar_init(&mma_done, 1);
        mbar_init(&sums_full, 8 * max(1, (int)cluster_size() - 1));
        mbar_init(&sums_empty, 8);
        mbar_init(&half_full, 8);
        mbar_init(&half_empty, 8);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMSums) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&s_tmem)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    cluster_meet();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const int size = (int)cluster_size(), rank = (int)cluster_rank(), mine = (int)blockIdx.x / size;
    const Found f = find<kMThreads>(kv.B, [&](int b) { return (int64_t)mass_shares(a, b); },
                                    [&](int64_t) { return (int64_t)mine / kv.heads; });
    MassWalk walk{f.before, f.b < 0 ? kv.B : f.b, mine, (int)gridDim.x / size, rank, size};
    // Every role walks the CTA's items by itself, as far ahead as the barriers let it: a
    // tile of rows is number g + i of all the CTA's, an item of keys number n.  (One loop,
    // so that the walk's instructions are fetched once.)
    MassItem it;
    uint32_t g = 0, n = 0;
    bool ok = true;
    const int w = warp - kMSums - 1;
    int64_t last = -1;  // tile of rows that this warp copied
    const TileCopy<DP> tile(lane, kv.dim);
    for (; ok && walk.next(a, it); g += (uint32_t)it.nt) {
        if (warp < kMSums) {
            // ------------------------------------------------ sums
            const int tile = (warp >> 2) & 1, odd = warp >> 3, own = tile * kCM + (warp & 3) * 32 + lane;
            const uint64_t scale_2 = pair(a.scale2, a.scale2);
            const uint32_t ts = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(tile * 2 * kCN);
            const int key = it.k0 + own;
            const bool real = key < it.len;
            const int lo = real ? it.first_row(a, key) : 0, hi = real ? it.last_row(a, key) : INT_MAX;
            // (looked up while the first tile is on its way, and read while it is summed)
            uint32_t slot, nth;
            kv.ps.divmod((uint32_t)key, nth, slot);
            const int page = real && rank == 0 && !odd ? kv.table[it.b * kv.table_stride + nth] : -1;
            float *mass = nullptr, was = 0.0f;
            auto look = [&] {
                if (mass || page < 0 || page >= kv.pages) return;
                mass = kv.mass_at(page, (int)slot, it.hk);
                was = *mass;
            };
            uint64_t sum[2] = {0u, 0u};
            for (int i = (int)((g + odd) & 1); i < it.nt; i += 2) {
                const uint32_t x = g + i;
                ok = mbar_wait_warp(&shift_full[x % kShifts], (x / kShifts) & 1, err, kWaitNs) &&
                     mbar_wait_warp(&s_full[tile][x & 1], (x >> 1) & 1, err, kWaitNs);
                if (!ok) break;
                tc_fence_after();
                look();
                const int q0 = it.r0 + i * kCM;
                const bool masked = __any_sync(kFull, q0 < lo || hi - kCM < q0);
                // some of the scores at a time, the next ones on their way
                constexpr int kPart = 16;
                float s[2][kPart];
                tmem_ld16_async(ts + (x & 1) * kCN, s[0]);
#pragma unroll
                for (int c = 0; c < kCN / kPart; ++c) {
                    float *v = s[c & 1];
                    tmem_ld_wait();
                    if (c + 1 < kCN / kPart) {
                        tmem_ld16_async(ts + (x & 1) * kCN + kPart * (c + 1), s[(c + 1) & 1]);
                    } else {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&s_empty[tile][x & 1]);
                    }
                    if (masked) {
                        // bits of the rows that see this key
                        const int from = lo - q0 - kPart * c, to = hi - q0 - kPart * c;
                        constexpr uint32_t kAll = (1u << kPart) - 1u;
                        uint32_t see = to >= kPart ? kAll : to <= 0 ? 0u : (1u << to) - 1u;
                        if (from > 0) see = from >= kPart ? 0u : see & ~((1u << from) - 1u);
                        if (__any_sync(kFull, see != kAll)) {
#pragma unroll
                            for (int e = 0; e < kPart; ++e) v[e] = see >> e & 1 ? v[e] : -INFINITY;
                        }
                    }
                    const ulonglong2 *sh = reinterpret_cast<const ulonglong2 *>(s_shift[x % kShifts] + kPart * c);
#pragma unroll
                    for (int e = 0; e < kPart; e += 4) {
                        const ulonglong2 z = sh[e / 4];
                        float p, q;
                        unpair(fma2(pair(v[e], v[e + 1]), scale_2, z.x), p, q);
                        sum[0] = add2(sum[0], pair(exp2_fast(p), exp2_fast(q)));
                        unpair(fma2(pair(v[e + 2], v[e + 3]), scale_2, z.y), p, q);
                        sum[1] = add2(sum[1], pair(exp2_fast(p), exp2_fast(q)));
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&shift_empty[x % kShifts]);
            }
            float p, q;
            unpair(add2(sum[0], sum[1]), p, q);
            p += q;
            if (!ok) break;
            const uint32_t turn = n++;
            if (odd) {
                ok = turn == 0 || mbar_wait_warp(&half_empty, (turn - 1) & 1, err, kWaitNs);
                if (!ok) break;
                s_half[own] = p;
                __syncwarp();
                if (lane == 0) mbar_arrive(&half_full);
                continue;
            }
            look();
            ok = mbar_wait_warp(&half_full, turn & 1, err, kWaitNs);
            if (!ok) break;
            p += s_half[own];
            __syncwarp();
            if (lane == 0) mbar_arrive(&half_empty);
            if (rank > 0) {  // to the first, once it has taken the item before
                ok = turn == 0 || peer_wait(&sums_empty, (turn - 1) & 1, err);
                if (!ok) break;
                peer_store(peer_addr(&s_sums[rank - 1][own], 0), p);
                __syncwarp();
                if (lane == 0) peer_arrive(peer_addr(&sums_full, 0));
                continue;
            }
            if (size > 1) {
                ok = peer_wait(&sums_full, turn & 1, err);
                if (!ok) break;
                for (int r = 1; r < size; ++r) p += s_sums[r - 1][own];
                __syncwarp();
                if (lane < size - 1) peer_arrive(peer_addr(&sums_empty, (uint32_t)lane + 1));
            }
            if (mass) *mass = was + p;
        } else if (it.nt == 0) {
            continue;
        } else if (warp == kMSums) {
            // ------------------------------------------------ MMA issuer
            const uint32_t idesc = chunk_idesc<T>(kCN) | (a.negative ? 1u << 13 : 0u);
            ok = mbar_wait_warp(&k_full[n % kItems], (n / kItems) & 1, err, kWaitNs);
            for (int i = 0; i < it.nt && ok; ++i) {
                const uint32_t x = g + i;
                ok = mbar_wait_warp(&full[x % kSt], (x / kSt) & 1, err, kWaitNs);
                const uint64_t bd = sw128_desc(ring + (x % kSt) * C::kTileBytes);
                for (int t = 0; t < 2 && ok; ++t) {
                    ok = mbar_wait_warp(&s_empty[t][x & 1], ((x >> 1) & 1) ^ 1, err, kWaitNs);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t ad = sw128_desc(base + (2 * (n % kItems) + t) * C::kTileBytes);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            const uint32_t off = (uint32_t)((k >> 2) * (C::kSlab >> 4) + (k & 3) * 2);
                            mma_ss(tmem + (2 * t + (x & 1)) * kCN, ad + off, bd + off, idesc, k > 0);
                        }
                        commit(&s_full[t][x & 1]);
                    }
                    __syncwarp();
                }
                if (elect_one()) commit(&empty[x % kSt]);
                __syncwarp();
            }
            if (elect_one()) commit(&k_empty[n % kItems]);
            __syncwarp();
            ++n;
        } else {
            // ------------------------------------------------ copies
            if (w == 2) {  // the third takes the keys
                const uint32_t item = n % kItems;
                if (n >= kItems && !mbar_wait_warp(&k_empty[item], ((n / kItems) & 1) ^ 1, err, kWaitNs)) break;
                int copied = 0;
                for (int t = 0; t < 2; ++t) {
                    const uint32_t dst = base + (2 * item + t) * C::kTileBytes;
                    const int key0 = it.k0 + t * kCM;
                    if (a.box && tile.fetch(dst, &k_map, a.box, kv, it.b, it.hk, key0, it.len, &k_full[item])) continue;
                    tile.copy(dst, kv.K, [&](int rr, int64_t &off) {
                        const bool is = key_place(kv, it.b, it.len, key0 + rr, kv.k_page, kv.k_slot, off);
                        off += it.hk * kv.k_head;
                        return is;
                    });
                    ++copied;
                }
                if (copied) tile.arrive(&k_full[item], copied);
                ++n;
                continue;
            }
            // the others tiles of rows in turn, with their lse2 (rows past the end are masked)
            for (int i = 0; i < it.nt; ++i) {
                const uint32_t x = g + i, round = x / kSt;
                if ((int)(x & 1) != w) continue;
                static_assert(kSt == kShifts && kSt % 2 == 0);
                // (each barrier has one warp that waits for it, which it then is never two phases
                // ahead of)
                ok = round == 0 || mbar_wait_warp(&empty[x % kSt], (round & 1) ^ 1, err, kWaitNs);
                if (!ok) break;
                const int q0 = it.r0 + i * kCM;
                const uint32_t dst = ring + (x % kSt) * C::kTileBytes;
                last = x;
                if (a.q_box) {
                    if (lane == 0) {
                        mbar_arrive_tx(&full[x % kSt], C::kTileBytes);
#pragma unroll
                        for (int s = 0; s < C::kSlabs; ++s)
                            tma_load_3d(dst + s * C::kSlab, &q_map, 64 * s, it.hk * a.G, it.t0 + q0 / a.G, &full[x % kSt]);
                    }
                    __syncwarp();
                } else {
                    tile.copy(dst, static_cast<const char *>(j.q), [&](int rr, int64_t &off) {
                        uint32_t t, h;
                        a.group.divmod((uint32_t)(q0 + rr), t, h);
                        off = (int64_t)(it.t0 + (int)t) * j.q_token + (int64_t)(it.hk * a.G + (int)h) * j.q_head;
                        return q0 + rr < it.rows;
                    });
                    tile.arrive(&full[x % kSt]);
                }
                ok = round == 0 || mbar_wait_warp(&shift_empty[x % kShifts], (round & 1) ^ 1, err, kWaitNs);
                if (!ok) break;
                const float *lse2 = j.lse2 + (int64_t)it.t0 * j.Hq + it.hk * a.G;
                const uint32_t sh = smem_addr(s_shift[x % kShifts]);
#pragma unroll
                for (int y = 0; y < kCM / 32; ++y) {
                    const int rr = 32 * y + lane, r = min(q0 + rr, it.rows - 1);
                    uint32_t t, h;
                    a.group.divmod((uint32_t)r, t, h);
                    copy4(sh + 4 * rr, lse2 + (int64_t)t * j.Hq + h, true);
                }
                copy_arrive(&shift_full[x % kShifts]);
            }
            ++n;
        }
    }
    if (warp == kMSums) {
        // every MMA is through before the memory that it reads goes
        if (elect_one()) commit(&mma_done);
        __syncwarp();
        mbar_wait_warp(&mma_done, 0, err, kWaitNs);
    } else if (warp > kMSums) {
        copy_commit();
        copy_wait<0>();
        // copies in flight complete before the CTA may exit: of this warp's tiles the last
        // two, whose places nothing has filled since
        static_assert(kSt == 4, "every second tile, two of a round");
        for (int64_t y = last; w < 2 && y >= 0 && y > last - 4; y -= 2)
            mbar_wait_warp(&full[y % kSt], (uint32_t)(y / kSt) & 1, err, kWaitNs);
        for (uint32_t y = n > kItems ? n - kItems : 0; w == 2 && y < n; ++y)
            mbar_wait_warp(&k_full[y % kItems], (y / kItems) & 1, err, kWaitNs);
    }
    tc_fence_before();
    __syncthreads();
    cluster_meet();  // no peer's store or arrival is on its way here
    if (warp == kMSums) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
    end_after(a.j.beside);
}

template <typename T, int DP>
cudaError_t mass(const AttendJob &j, const KvView &kv, cudaStream_t s) {
    MassArgs a{};
    a.j = j;
    a.kv = kv;
    a.scale2 = std::max(std::fabs(j.scale) * kLog2e, 1e-37f);
    a.G = j.Hq / kv.heads;
    a.negative = j.scale < 0.0f;
    a.group = FastDiv((uint32_t)a.G);
    a.heads = FastDiv((uint32_t)kv.heads);
    CUtensorMap maps[2] = {};
    a.box = page_box(kv);
    if (a.box && page_map(&maps[0], kv, false, j.type, a.box) != cudaSuccess) a.box = 0;
    a.q_box = rows_map(&maps[1], j, kv, a.G);
    uint32_t *err = library_error_word();
    if (!err) return cudaErrorUnknown;
    int dev = 0, sms = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d;
    const int64_t items = (int64_t)kv.B * kv.heads * ((room + kMKeys - 1) / kMKeys);
    const int64_t tiles = ((int64_t)kv.max_new * a.G + kCM - 1) / kCM;
    // CTAs of a cluster: as many as let all be through first, in turns of items with as
    // many tiles of rows each, and as long as three beside them (four with peers).  (2051
    // tokens of 8 heads a key head over themselves: 194 us a call with a CTA an item, 95
    // with clusters; 83 now.)
    int share = 1;
    int64_t best = INT64_MAX;
    for (int n = 1; n <= kMostShare; n *= 2) {
        const int64_t at = std::max(1, sms / n), cost = (items + at - 1) / at * ((tiles + n - 1) / n + (n > 1 ? 4 : 3));
        if (cost < best) best = cost, share = n;
    }
    const cudaError_t e = func_attr(reinterpret_cast<const void *>(k_mass<T, DP>),
                                    cudaFuncAttributeMaxDynamicSharedMemorySize, Mass<DP>::kSmem);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)(std::min<int64_t>(items, std::max(1, sms / share)) * share);
    return launch_cluster(k_mass<T, DP>, dim3(grid), share, kMThreads, Mass<DP>::kSmem, s, a, maps[0], maps[1], err);
}

}  // namespace

cudaError_t launch_attention_mass(const AttendJob &j, const KvView &kv, cudaStream_t s) {
    if (j.type == PVMVMD_BF16) return kv.dim <= 64 ? mass<__nv_bfloat16, 64>(j, kv, s) : mass<__nv_bfloat16, 128>(j, kv, s);
    return kv.dim <= 64 ? mass<__half, 64>(j, kv, s) : mass<__half, 128>(j, kv, s);
}

}  // namespace pv
